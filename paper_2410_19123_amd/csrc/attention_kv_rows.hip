// Attention over the 8-bit cache for few query rows per request: decode steps
// and drafted tokens (attention_kv.hpp has the mathematics).
//
// A pair is (request, tile of 16 NT rows, key head); its work is the blocks of
// 64 tokens that the request sees.  The call's blocks, pair after pair, are
// dealt to the workgroups in equal contiguous shares, so that one long request
// among short ones, or few requests, fill the chip alike.  A share may begin
// and end inside a pair: those ends are partial results (m, l, sums) in the
// workspace, at most two per workgroup, and a second launch joins them; a pair
// inside one share is written at once.
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
// Workgroups a call is dealt to, and the least blocks of a share.
constexpr int kShares = 1024;
constexpr int kMinShare = 4;

template <int D, int NT>
constexpr int kPartFloats = NT * (16 * D + 128);

// Workspace: [0] blocks per share, [1 .. R + 1] first block of each request's
// pairs (int64), then two parts per workgroup.
size_t plan_bytes(int64_t R) { return (size_t)round_up((R + 2) * 8, 256); }

struct Plan {
    int64_t weight;  // blocks of all the request's pairs
    int tiles;
    int blocks;      // of each pair
};

template <int NT>
__device__ __forceinline__ Plan plan_of(const KvAttnArgs& a, const KvRequest& q) {
    Plan p;
    p.tiles = (int)(((int64_t)q.n * a.G + 16 * NT - 1) / (16 * NT));
    p.blocks = q.block1 - q.block0;
    p.weight = (int64_t)p.tiles * a.c.Hk * p.blocks;
    return p;
}

__device__ __forceinline__ int64_t wave_scan64(int64_t v, int lane) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int64_t u = __shfl_up(v, off, 64);
        if (lane >= off) v += u;
    }
    return v;
}

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

    // Part layout, per lane: sums [NT][D / 16][64] float4, then m and l
    // [NT][2][64].
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
};

// 16 dims of one row tile to bf16 at the rows they belong to.
template <int D, int NT>
__device__ __forceinline__ void store_rows(const KvAttnArgs& a, const KvRequest& q, int tile, int h,
                                           int nt, int d, const f32x4 acc, float l) {
    const int lane = threadIdx.x & 63, col = lane & 15, qt = lane >> 4;
    const int i = (tile * NT + nt) * 16 + col;
    if (i >= q.n * a.G) return;
    const int tok = i / a.G, head = h * a.G + i - tok * a.G;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    uint2 w;
    w.x = (uint32_t)f32_to_bf16(acc[0] * inv) | ((uint32_t)f32_to_bf16(acc[1] * inv) << 16);
    w.y = (uint32_t)f32_to_bf16(acc[2] * inv) | ((uint32_t)f32_to_bf16(acc[3] * inv) << 16);
    *reinterpret_cast<uint2*>(a.o + (q.row0 + tok) * a.ld_o + (int64_t)head * D + d * 16 + 4 * qt) = w;
}

template <int KT, int D, int NT>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2)))
void k_attention_rows(KvAttnArgs a, int64_t* __restrict__ plan, float* __restrict__ parts) {
    __shared__ __attribute__((aligned(16))) float xs[2 * kPartFloats<D, NT>];
    __shared__ int64_t sums[kWaves];
    __shared__ int64_t at_base, at_req;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int64_t R = a.c.R;

    // Blocks of the whole call, then this workgroup's share of them.
    int64_t mine = 0;
    for (int64_t r = tid; r < R; r += kThreads) mine += plan_of<NT>(a, kv_request(a, r)).weight;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) mine += __shfl_xor(mine, off, 64);
    if (lane == 0) sums[wv] = mine;
    __syncthreads();
    int64_t total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += sums[w];
    int64_t share = (total + gridDim.x - 1) / gridDim.x;
    share = share < kMinShare ? kMinShare : share;
    const int64_t w0 = (int64_t)blockIdx.x * share;
    const int64_t w1 = w0 + share < total ? w0 + share : total;
    // The request that w0 lies in (workgroup 0 also writes the plan down).
    if (blockIdx.x == 0 && tid == 0) plan[0] = share;
    if (w0 >= total && blockIdx.x != 0) return;
    int64_t run = 0;
    for (int64_t r0 = 0; r0 < R; r0 += kThreads) {
        const int64_t r = r0 + tid;
        const int64_t w = r < R ? plan_of<NT>(a, kv_request(a, r)).weight : 0;
        const int64_t incl = wave_scan64(w, lane);
        __syncthreads();
        if (lane == 63) sums[wv] = incl;
        __syncthreads();
        int64_t base = run + incl - w;
        int64_t all = 0;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            if (k < wv) base += sums[k];
            all += sums[k];
        }
        if (r < R && w0 >= base && w0 < base + w) {
            at_base = base;
            at_req = r;
        }
        if (blockIdx.x == 0 && r < R) plan[1 + r] = base;
        run += all;
        if (blockIdx.x != 0 && run > w0) break;
    }
    if (w0 >= total) return;
    __syncthreads();

    int64_t r = at_req, base = at_base;
    KvRequest q = kv_request(a, r);
    Plan p = plan_of<NT>(a, q);
    RowsState<KT, D, NT> st;
    for (int64_t w = w0; w < w1;) {
        while (w >= base + p.weight) {  // ends: w < total
            base += p.weight;
            q = kv_request(a, ++r);
            p = plan_of<NT>(a, q);
        }
        const int pair = (int)((w - base) / p.blocks);
        const int b0 = (int)((w - base) - (int64_t)pair * p.blocks);
        const int left = p.blocks - b0;
        const int nb = w1 - w < left ? (int)(w1 - w) : left;
        const int tile = pair / a.c.Hk, h = pair - tile * a.c.Hk;
        st.start(a, q, tile, h);
        // Wave wv takes blocks wv, wv + 4, ...; lane i holds the block number
        // and scales of the wave's i-th of the next 64.
        for (int i0 = wv; i0 < nb; i0 += 64 * kWaves) {
            const int i = i0 + lane * kWaves;
            int blk = -1;
            float ks = 0.0f, vs = 0.0f;
            if (i < nb) {
                blk = (int)kv_block_of(a.c.table, a.c.max_blocks, a.c.n_blocks, r, q.block0 + b0 + i);
                if (blk >= 0) {
                    const float2 sc = *reinterpret_cast<const float2*>(
                        a.c.scales + ((int64_t)blk * a.c.Hk + h) * 2);
                    ks = sc.x;
                    vs = sc.y;
                }
            }
            const int cnt = (nb - i0 + kWaves - 1) / kWaves;
            for (int k = 0; k < (cnt < 64 ? cnt : 64); ++k) {
                const int bk = __builtin_amdgcn_readlane(blk, k);
                if (bk < 0) continue;
                const float ksk = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks), k));
                const float vsk = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs), k));
                st.block(a.c.codes + ((int64_t)bk * a.c.Hk + h) * 2 * kKvBlock * D, ksk, vsk,
                         (q.block0 + b0 + i0 + k * kWaves) * kKvBlock, q.len);
            }
        }
        st.finish();
        // Waves 2 and 3 into 0 and 1, then 1 into 0.
        __syncthreads();
        if (wv >= 2) st.put(xs + (wv - 2) * kPartFloats<D, NT>);
        __syncthreads();
        if (wv < 2) st.join(xs + wv * kPartFloats<D, NT>);
        __syncthreads();
        if (wv == 1) st.put(xs);
        __syncthreads();
        if (wv == 0) {
            st.join(xs);
            if (nb == p.blocks) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int d = 0; d < D / 16; ++d)
                        store_rows<D, NT>(a, q, tile, h, nt, d, st.acc[nt][d], st.l[nt]);
            } else {
                st.put(parts + ((int64_t)blockIdx.x * 2 + (b0 == 0 ? 1 : 0)) * kPartFloats<D, NT>);
            }
        }
        w += nb;
    }
}

// Joins the parts of each pair that several workgroups shared, and zeroes the
// rows of a request that sees no block.  One workgroup per (row tile slot,
// head); tile j of request r is slot floor(offsets[r] G / rows) + r + j, which
// needs no sum over the requests and leaves some slots empty.
template <int D, int NT>
__global__ __launch_bounds__(kThreads) void k_attention_join(KvAttnArgs a,
                                                             const int64_t* __restrict__ plan,
                                                             const float* __restrict__ parts) {
    constexpr int kRows = 16 * NT;
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int h = blockIdx.y;
    const int64_t slot = blockIdx.x;
    // The last request whose first slot is at most this one.
    int64_t lo = 0, n = a.c.R;
    while (n > 1) {
        const int64_t step = (n + 63) / 64, i = lane * step;
        const bool le = i < n && (int64_t)a.c.offsets[lo + i] * a.G / kRows + lo + i <= slot;
        const int below = __popcll(__ballot(le));
        const int64_t skip = below > 0 ? (int64_t)(below - 1) * step : 0;
        lo += skip;
        n = n - skip < step ? n - skip : step;
    }
    const KvRequest q = kv_request(a, lo);
    const Plan p = plan_of<NT>(a, q);
    const int64_t tl = slot - ((int64_t)a.c.offsets[lo] * a.G / kRows + lo);
    if (tl < 0 || tl >= p.tiles) return;
    const int tile = (int)tl;
    if (p.blocks == 0) {
        const f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int k = wv; k < NT * (D / 16); k += kWaves)
            store_rows<D, NT>(a, q, tile, h, k / (D / 16), k % (D / 16), z, 0.0f);
        return;
    }
    const int64_t share = plan[0];
    const int64_t s = plan[1 + lo] + ((int64_t)tile * a.c.Hk + h) * p.blocks, e = s + p.blocks;
    const int64_t g0 = s / share, g1 = (e - 1) / share;
    if (g0 == g1) return;
    auto part = [&](int64_t g) {
        return parts + (g * 2 + (g == g0 ? 1 : 0)) * kPartFloats<D, NT>;
    };
    for (int nt = 0; nt < NT; ++nt) {
        float m = -INFINITY;
        for (int64_t g = g0; g <= g1; ++g)
            m = fmaxf(m, (part(g) + NT * 16 * D + nt * 128)[lane]);
        const float base = m == -INFINITY ? 0.0f : m;
        float l = 0.0f;
        constexpr int ND = D / 16 / kWaves;  // 16-dim tiles per wave
        f32x4 acc[ND];
#pragma unroll
        for (int d = 0; d < ND; ++d) acc[d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int64_t g = g0; g <= g1; ++g) {
            const float* pp = part(g);
            const float* ml = pp + NT * 16 * D + nt * 128;
            const float f = __builtin_amdgcn_exp2f(ml[lane] - base);
            l = fmaf(ml[64 + lane], f, l);
#pragma unroll
            for (int d = 0; d < ND; ++d)
                acc[d] += reinterpret_cast<const f32x4*>(pp)[(nt * (D / 16) + wv * ND + d) * 64 + lane] * f;
        }
#pragma unroll
        for (int d = 0; d < ND; ++d)
            store_rows<D, NT>(a, q, tile, h, nt, wv * ND + d, acc[d], l);
    }
}

template <int KT, int D, int NT>
hipError_t run_rows(const KvAttnArgs& a, hipStream_t s) {
    int64_t* plan = reinterpret_cast<int64_t*>(a.ws);
    float* parts = reinterpret_cast<float*>(reinterpret_cast<char*>(a.ws) + plan_bytes(a.c.R));
    k_attention_rows<KT, D, NT><<<kShares, kThreads, 0, s>>>(a, plan, parts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)(a.c.T * a.G / (16 * NT) + a.c.R), (unsigned)a.c.Hk);
    k_attention_join<D, NT><<<grid, kThreads, 0, s>>>(a, plan, parts);
    return hipGetLastError();
}

template <int KT, int D>
hipError_t rows_of(const KvAttnArgs& a, hipStream_t s) {
    return run_rows<KT, D, 1>(a, s);
}

}  // namespace

size_t kv_attention_workspace(int64_t T, int64_t R, int H, int Hk, int D, int64_t max_blocks) {
    (void)T;
    (void)H;
    (void)Hk;
    (void)max_blocks;
    return plan_bytes(R) + (size_t)kShares * 2 * 4 * (16 * D + 128);
}

hipError_t launch_kv_attention(readme_kv_type kt, const KvAttnArgs& a, hipStream_t s) {
    const bool i8 = kt == README_KV_I8;
    switch (a.c.D) {
        case 64: return i8 ? rows_of<README_KV_I8, 64>(a, s) : rows_of<README_KV_E4M3, 64>(a, s);
        case 128: return i8 ? rows_of<README_KV_I8, 128>(a, s) : rows_of<README_KV_E4M3, 128>(a, s);
        case 256: return i8 ? rows_of<README_KV_I8, 256>(a, s) : rows_of<README_KV_E4M3, 256>(a, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace readme
