// Attention over the 8-bit cache for few query rows per request: decode steps
// and drafted tokens (attention_kv.hpp has the mathematics).
//
//   The four waves of a workgroup take its blocks in turn, each straight from
// global memory to registers with no LDS and no barrier:
//     S^T = K Q^T   16x16x32 MFMA; a lane gets 16 scores of one row, the 16
//                   tokens whose codes it loads for V, so P stays in its
//                   registers;
//     O^T += V^T P^T.
// The waves' sums meet in LDS at the end of a pair.
#include <math.h>

#include "attention_kv.hpp"

namespace readme {

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr int kMinShare = 4;

template <int D, int NT>
constexpr int kXchgFloats = NT * (16 * D + 128);

// One wave's running result over the blocks it takes.
template <int KT, int D, int NT>
struct RowsState {
    f16x8 qf[NT][D / 32];
    f32x4 acc[NT][D / 16];
    float m[NT], l[NT], cq[NT];
    int lo[NT], hi[NT];
    float vref;
    int min_hi, max_lo;

    __device__ __forceinline__ void start(const KvAttnArgs& a, const KvRequest& q, int tile, int h) {
        const int lane = threadIdx.x & 63, col = lane & 15, qt = lane >> 4;
        min_hi = 0x7fffffff;
        max_lo = 0;
        vref = 0.0f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int i = (tile * NT + nt) * 16 + col;
            const bool real = i < q.n * a.G;
            const int tok = real ? i / a.G : 0;
            const int head = h * a.G + (real ? i - tok * a.G : 0);
            const uint16_t* row = a.q + (q.row0 + tok) * a.ld_q + (int64_t)head * D;
            float x[D / 32][8];
            float big = 0.0f;
#pragma unroll
            for (int f = 0; f < D / 32; ++f) {
                uint4 w = make_uint4(0u, 0u, 0u, 0u);
                if (real) w = *reinterpret_cast<const uint4*>(row + (f >> 1) * 64 + qt * 16 + (f & 1) * 8);
                const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[f][2 * e] = bf16_lo(v[e]);
                    x[f][2 * e + 1] = bf16_hi(v[e]);
                    big = fmaxf(big, fmaxf(fabsf(x[f][2 * e]), fabsf(x[f][2 * e + 1])));
                }
            }
            big = fmaxf(big, __shfl_xor(big, 16, 64));
            big = fmaxf(big, __shfl_xor(big, 32, 64));
            float up, down;
            row_power(big, up, down);
            cq[nt] = a.score * down;
#pragma unroll
            for (int f = 0; f < D / 32; ++f)
#pragma unroll
                for (int e = 0; e < 8; ++e) qf[nt][f][e] = (_Float16)(x[f][e] * up);
            row_keys(a, q.len, (int64_t)q.len - q.n + tok, lo[nt], hi[nt]);
            if (real) {
                min_hi = hi[nt] < min_hi ? hi[nt] : min_hi;
                max_lo = lo[nt] > max_lo ? lo[nt] : max_lo;
            }
            m[nt] = -INFINITY;
            l[nt] = 0.0f;
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
#pragma unroll
                for (int i2 = 0; i2 < 4; ++i2) acc[nt][d][i2] = 0.0f;
        }
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) {
            const int u = __shfl_xor(min_hi, off, 64), w = __shfl_xor(max_lo, off, 64);
            min_hi = u < min_hi ? u : min_hi;
            max_lo = w > max_lo ? w : max_lo;
        }
    }

    // The 64 tokens of a block, token 0 at position j0.
    __device__ __forceinline__ void block(const uint8_t* kc, float ks, float vs, int j0, int len) {
        const int lane = threadIdx.x & 63, col = lane & 15, qt = lane >> 4;
        uint4 kf[4][D / 64], vf[D / 16];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int tok = 16 * (col >> 2) + 4 * t + (col & 3);
#pragma unroll
            for (int f = 0; f < D / 64; ++f)
                kf[t][f] = *reinterpret_cast<const uint4*>(
                    kc + (((tok >> 5) * (D / 16) + 4 * f + qt) * 32 + (tok & 31)) * 16);
        }
        const uint8_t* vc = kc + kKvBlock * D;
#pragma unroll
        for (int d = 0; d < D / 16; ++d)
            vf[d] = *reinterpret_cast<const uint4*>(vc + ((qt >> 1) * D + d * 16 + col) * 32 +
                                                    (qt & 1) * 16);
        if (j0 + kKvBlock > len) {
#pragma unroll
            for (int d = 0; d < D / 16; ++d) vf[d] = keep_tokens(vf[d], len - j0 - 16 * qt);
        }

        f32x4 s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int t = 0; t < 4; ++t) s[nt][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int f = 0; f < D / 64; ++f) {
                const f16x8 k0 = cvt8<KT>(kf[t][f].x, kf[t][f].y);
                const f16x8 k1 = cvt8<KT>(kf[t][f].z, kf[t][f].w);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    s[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, qf[nt][2 * f], s[nt][t], 0, 0, 0);
                    s[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, qf[nt][2 * f + 1], s[nt][t], 0, 0, 0);
                }
            }

        // Units of the sums: the largest value scale so far.
        if (vs > vref) {
            const float f = vref / vs;
            vref = vs;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int d = 0; d < D / 16; ++d) acc[nt][d] *= f;
        }
        float log_r, inv_r;
        value_ratio(vs, vref, log_r, inv_r);

        const bool masked = j0 + kKvBlock > min_hi || j0 < max_lo;
        f16x8 pf[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float c = cq[nt] * ks;
            // score (t, i) is token j0 + 16 qt + 4 t + i
            const int a0 = lo[nt] - j0 - 16 * qt, a1 = hi[nt] - j0 - 16 * qt;
            float mx = -INFINITY;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (masked && (4 * t + i < a0 || 4 * t + i >= a1)) s[nt][t][i] = -INFINITY;
                    mx = fmaxf(mx, s[nt][t][i]);
                }
            if (__any(mx * c > m[nt] + kLazy)) {
                float t = mx * c;
                t = fmaxf(t, __shfl_xor(t, 16, 64));
                t = fmaxf(t, __shfl_xor(t, 32, 64));
                const float mn = fmaxf(m[nt], t);
                const float f = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[nt] - mn);
                m[nt] = mn;
                l[nt] *= f;
#pragma unroll
                for (int d = 0; d < D / 16; ++d) acc[nt][d] *= f;
            }
            const float b = log_r + kUp - m[nt];
            float sum = 0.0f;
            uint32_t pw[8];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                float p[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[i] = __builtin_amdgcn_exp2f(fmaf(s[nt][t][i], c, b));
                    if (masked && (4 * t + i < a0 || 4 * t + i >= a1)) p[i] = 0.0f;
                    sum += p[i];
                }
                pw[2 * t] = pack_f16(p[0], p[1]);
                pw[2 * t + 1] = pack_f16(p[2], p[3]);
            }
            l[nt] = fmaf(sum, inv_r, l[nt]);
            pf[nt][0] = __builtin_bit_cast(f16x8, u32x4v{pw[0], pw[1], pw[2], pw[3]});
            pf[nt][1] = __builtin_bit_cast(f16x8, u32x4v{pw[4], pw[5], pw[6], pw[7]});
        }
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            const f16x8 v0 = cvt8<KT>(vf[d].x, vf[d].y);
            const f16x8 v1 = cvt8<KT>(vf[d].z, vf[d].w);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                acc[nt][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pf[nt][0], acc[nt][d], 0, 0, 0);
                acc[nt][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pf[nt][1], acc[nt][d], 0, 0, 0);
            }
        }
    }

    // l over the whole row, sums in units of one.
    __device__ __forceinline__ void finish() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            l[nt] += __shfl_xor(l[nt], 16, 64);
            l[nt] += __shfl_xor(l[nt], 32, 64);
#pragma unroll
            for (int d = 0; d < D / 16; ++d) acc[nt][d] *= vref;
        }
    }

    // In LDS, between the waves: sums [NT][D / 16][64 lanes] float4, then m and l
    // [NT][2][64 lanes].
    __device__ __forceinline__ void put(float* part) const {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
                reinterpret_cast<f32x4*>(part)[(nt * (D / 16) + d) * 64 + lane] = acc[nt][d];
            float* ml = part + NT * 16 * D + nt * 128;
            ml[lane] = m[nt];
            ml[64 + lane] = l[nt];
        }
    }
    __device__ __forceinline__ void join(const float* part) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float* ml = part + NT * 16 * D + nt * 128;
            const float m1 = ml[lane], l1 = ml[64 + lane];
            const float mn = fmaxf(m[nt], m1);
            const float base = mn == -INFINITY ? 0.0f : mn;
            const float f0 = __builtin_amdgcn_exp2f(m[nt] - base);
            const float f1 = __builtin_amdgcn_exp2f(m1 - base);
            m[nt] = mn;
            l[nt] = l[nt] * f0 + l1 * f1;
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
                acc[nt][d] = acc[nt][d] * f0 +
                             reinterpret_cast<const f32x4*>(part)[(nt * (D / 16) + d) * 64 + lane] * f1;
        }
    }

    // The rows in bf16 where they belong.
    __device__ __forceinline__ void store(const KvAttnArgs& a, const KvRequest& q, int tile, int h) const {
        const int lane = threadIdx.x & 63, col = lane & 15, qt = lane >> 4;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int i = (tile * NT + nt) * 16 + col;
            if (i >= q.n * a.G) continue;
            const int tok = i / a.G, head = h * a.G + i - tok * a.G;
            uint16_t* row = a.o + (q.row0 + tok) * a.ld_o + (int64_t)head * D + 4 * qt;
            const float inv = l[nt] == 0.0f ? 0.0f : 1.0f / l[nt];
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                uint2 w;
                w.x = (uint32_t)f32_to_bf16(acc[nt][d][0] * inv) | ((uint32_t)f32_to_bf16(acc[nt][d][1] * inv) << 16);
                w.y = (uint32_t)f32_to_bf16(acc[nt][d][2] * inv) | ((uint32_t)f32_to_bf16(acc[nt][d][3] * inv) << 16);
                *reinterpret_cast<uint2*>(row + d * 16) = w;
            }
        }
    }
    __device__ __forceinline__ void store_part(float* part) const {
        const int lane = threadIdx.x & 63, col = lane & 15, qt = lane >> 4;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int i = nt * 16 + col;
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
                *reinterpret_cast<f32x4*>(part + i * D + d * 16 + 4 * qt) = acc[nt][d];
            if (qt == 0) {
                part[16 * NT * D + i] = m[nt];
                part[16 * NT * (D + 1) + i] = l[nt];
            }
        }
    }
};

template <int KT, int D, int NT>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2)))
void k_attention_rows(KvAttnArgs a, int64_t* __restrict__ plan, float* __restrict__ parts) {
    constexpr int kRows = 16 * NT;
    __shared__ __attribute__((aligned(16))) float xs[2 * kXchgFloats<D, NT>];
    __shared__ int64_t found[kWaves + 2];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    KvShare sh;
    if (!kv_share<kRows, kWaves>(a, kMinShare, plan, found, sh)) return;

    int64_t r = sh.r, base = sh.base;
    KvRequest q = kv_request(a, r);
    KvPlan p = kv_plan<kRows>(a, q);
    RowsState<KT, D, NT> st;
    for (int64_t w = sh.w0; w < sh.w1;) {
        while (w >= base + p.weight) {  // ends: w is below the sum of all weights
            base += p.weight;
            q = kv_request(a, ++r);
            p = kv_plan<kRows>(a, q);
        }
        const int pair = (int)((w - base) / p.blocks);
        const int b0 = (int)((w - base) - (int64_t)pair * p.blocks);
        const int left = p.blocks - b0;
        const int nb = sh.w1 - w < left ? (int)(sh.w1 - w) : left;
        const int tile = pair / a.c.Hk, h = pair - tile * a.c.Hk;
        st.start(a, q, tile, h);
        // Wave wv takes blocks wv, wv + 4, ...; lane i holds the block number
        // and scales of the wave's i-th of the next 64.
        for (int i0 = wv; i0 < nb; i0 += 64 * kWaves) {
            KvBlockRef mine;
            mine.blk = -1;
            if (i0 + lane * kWaves < nb)
                mine = kv_block_ref(a, r, q.block0 + b0 + i0 + lane * kWaves, h);
            const int cnt = (nb - i0 + kWaves - 1) / kWaves;
            for (int k = 0; k < (cnt < 64 ? cnt : 64); ++k) {
                const KvBlockRef b = kv_lane_ref(mine, k);
                if (b.blk < 0) continue;
                st.block(a.c.codes + ((int64_t)b.blk * a.c.Hk + h) * 2 * kKvBlock * D, b.ks, b.vs,
                         (q.block0 + b0 + i0 + k * kWaves) * kKvBlock, q.len);
            }
        }
        st.finish();
        // Waves 2 and 3 into 0 and 1, then 1 into 0.
        __syncthreads();
        if (wv >= 2) st.put(xs + (wv - 2) * kXchgFloats<D, NT>);
        __syncthreads();
        if (wv < 2) st.join(xs + wv * kXchgFloats<D, NT>);
        __syncthreads();
        if (wv == 1) st.put(xs);
        __syncthreads();
        if (wv == 0) {
            st.join(xs);
            if (nb == p.blocks)
                st.store(a, q, tile, h);
            else
                st.store_part(parts + ((int64_t)blockIdx.x * 2 + (b0 == 0 ? 1 : 0)) *
                                          kv_part_floats<D, kRows>);
        }
        w += nb;
    }
}

template <int KT, int D>
hipError_t rows_of(const KvAttnArgs& a, hipStream_t s) {
    int64_t* plan = reinterpret_cast<int64_t*>(a.ws);
    float* parts = reinterpret_cast<float*>(reinterpret_cast<char*>(a.ws) + kv_plan_bytes(a.c.R));
    k_attention_rows<KT, D, 1><<<kRowsShares, kThreads, 0, s>>>(a, plan, parts);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_rows(readme_kv_type kt, const KvAttnArgs& a, hipStream_t s) {
    const bool i8 = kt == README_KV_I8;
    switch (a.c.D) {
        case 64: return i8 ? rows_of<README_KV_I8, 64>(a, s) : rows_of<README_KV_E4M3, 64>(a, s);
        case 128: return i8 ? rows_of<README_KV_I8, 128>(a, s) : rows_of<README_KV_E4M3, 128>(a, s);
        case 256: return i8 ? rows_of<README_KV_I8, 256>(a, s) : rows_of<README_KV_E4M3, 256>(a, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace readme
