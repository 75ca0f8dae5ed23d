// Attention over the 8-bit cache for few query rows per request: decode steps
// and drafted tokens (attention_kv.hpp has the mathematics).
//
//   The waves of a workgroup take its blocks in turn, each straight from global
// memory to registers with no LDS and no barrier:
//     S^T = K Q^T   16x16x32 MFMA; a lane gets 16 scores of one row, of the 16
//                   tokens whose codes it loads for V, so P stays in its
//                   registers;
//     O^T += V^T P^T.
// A block's K registers are loaded with the next block's codes as soon as the
// scores have taken them, V's as soon as the sums have, so that 8 to 16 KB per
// wave are always on their way.  The waves' sums meet in LDS at the end of a
// pair.  Bound by the codes' stream: 8 requests of 60000 to 126000 tokens, 1.53
// GB, 260 us and 6 for the join of the shares (5.8 TB/s, 1.006 times the codes
// fetched); 32 x 32 heads on 2048 tokens, 538 MB, 94 us (5.7); 64 requests of 1 to
// 4096 tokens, 267 MB, 48 us from the last-level cache and 62 from memory, where
// the longest requests end alone; one request of 517 tokens 9 us, two dependent
// loads (table, scales), four blocks and the waves' join.  32 rows a pair instead
// of 16: the same times, and registers spilled at 128 dims.
#include <math.h>

#include "attention_kv.hpp"

namespace readme {

namespace {

constexpr int kRows = kRowsTile;
constexpr int kMinShare = 16;

// One wave's running result over the blocks it takes, for 16 rows.
template <int KT, int D>
struct RowsState {
    static constexpr int NK = D / 64;  // 16-byte pieces of K per lane and score tile
    static constexpr int ND = D / 16;  // 16-dim tiles
    f16x8 qf[2 * NK];
    f32x4 acc[ND];
    uint4 kf[4][NK], vf[ND];
    float m, l, cq, vref, log_vref;
    int lo, hi;          // keys this lane's row sees
    int min_hi, max_lo;  // over the rows

    // The lane's row of q, D / 4 elements of it; tok < 0 where there is none.
    __device__ __forceinline__ void fetch(const KvAttnArgs& a, const KvRequest& q, int64_t tile, int h,
                                          uint4 (&raw)[2 * NK], int& tok) {
        const int lane = threadIdx.x & 63, col = lane & 15, qt = lane >> 4;
        const int64_t i = tile * kRows + col;
        const bool real = i < (int64_t)q.n * a.G;
        const int t = real ? (int)i / a.G : 0;  // i < n G <= 2^27
        const int head = h * a.G + (real ? (int)i - t * a.G : 0);
        const uint16_t* row = a.q + (q.row0 + t) * a.ld_q + (int64_t)head * D;
        tok = real ? t : -1;
#pragma unroll
        for (int f = 0; f < 2 * NK; ++f) {
            raw[f] = make_uint4(0u, 0u, 0u, 0u);
            if (real)
                raw[f] =
                    *reinterpret_cast<const uint4*>(row + (f >> 1) * 64 + qt * 16 + (f & 1) * 8);
        }
    }

    __device__ __forceinline__ void start(const KvAttnArgs& a, const KvRequest& q,
                                          const uint4 (&raw)[2 * NK], int tok) {
        min_hi = 0x7fffffff;
        max_lo = 0;
        float big = 0.0f;
#pragma unroll
        for (int f = 0; f < 2 * NK; ++f) {
            const uint32_t v[4] = {raw[f].x, raw[f].y, raw[f].z, raw[f].w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                big = fmaxf(big, fmaxf(fabsf(bf16_lo(v[e])), fabsf(bf16_hi(v[e]))));
        }
        big = fmaxf(big, __shfl_xor(big, 16, 64));
        big = fmaxf(big, __shfl_xor(big, 32, 64));
        float up, down;
        row_power(big, up, down);
        cq = a.score * down;
#pragma unroll
        for (int f = 0; f < 2 * NK; ++f) {
            const uint32_t v[4] = {raw[f].x, raw[f].y, raw[f].z, raw[f].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                qf[f][2 * e] = (_Float16)(bf16_lo(v[e]) * up);
                qf[f][2 * e + 1] = (_Float16)(bf16_hi(v[e]) * up);
            }
        }
        const bool real = tok >= 0;
        row_keys(a, q.len, (int64_t)q.len - q.n + (real ? tok : 0), lo, hi);
        min_hi = real ? min(min_hi, hi) : min_hi;
        max_lo = real ? max(max_lo, lo) : max_lo;
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) {
            min_hi = min(min_hi, __shfl_xor(min_hi, off, 64));
            max_lo = max(max_lo, __shfl_xor(max_lo, off, 64));
        }
        min_hi = __builtin_amdgcn_readfirstlane(min_hi);
        max_lo = __builtin_amdgcn_readfirstlane(max_lo);
    }

    __device__ __forceinline__ void clear() {
        vref = log_vref = 0.0f;
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int d = 0; d < ND; ++d) acc[d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    __device__ __forceinline__ void load_k(const uint8_t* kc) {
        const int lane = threadIdx.x & 63, col = lane & 15, qt = lane >> 4;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int tok = 16 * (col >> 2) + 4 * t + (col & 3);
#pragma unroll
            for (int f = 0; f < NK; ++f)
                kf[t][f] = *reinterpret_cast<const uint4*>(
                    kc + (((tok >> 5) * (D / 16) + 4 * f + qt) * 32 + (tok & 31)) * 16);
        }
    }
    __device__ __forceinline__ void load_v(const uint8_t* kc) {
        const int lane = threadIdx.x & 63, col = lane & 15, qt = lane >> 4;
        const uint8_t* vc = kc + kKvBlock * D;
#pragma unroll
        for (int d = 0; d < ND; ++d)
            vf[d] = *reinterpret_cast<const uint4*>(vc + ((qt >> 1) * D + d * 16 + col) * 32 +
                                                    (qt & 1) * 16);
    }

    // The block held in kf and vf, its token 0 at position j0; `next` is the
    // block whose codes take its place.
    __device__ __forceinline__ void block(float ks, float vs, int j0, int len, const uint8_t* next) {
        const int qt = (threadIdx.x & 63) >> 4;
        f32x4 s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            s[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int f = 0; f < NK; ++f) {
                const f16x8 k0 = cvt8<KT>(kf[t][f].x, kf[t][f].y);
                const f16x8 k1 = cvt8<KT>(kf[t][f].z, kf[t][f].w);
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, qf[2 * f], s[t], 0, 0, 0);
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, qf[2 * f + 1], s[t], 0, 0, 0);
            }
        }
        load_k(next);

        const bool edge = j0 + kKvBlock > min_hi || j0 < max_lo;
        value_unit(vs, !edge || sees_block(lo, hi, j0), vref, log_vref, acc, [](float x) {
            x = fmaxf(x, __shfl_xor(x, 16, 64));
            return fmaxf(x, __shfl_xor(x, 32, 64));
        });
        float log_r, inv_r;
        value_ratio(vs, log_vref, log_r, inv_r);

        const float c = score_factor(cq, ks);
        // score k = 4 t + i of the lane is token j0 + 16 qt + k
        float z[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) z[k] = s[k >> 2][k & 3];
        const int a0 = lo - j0 - 16 * qt, a1 = hi - j0 - 16 * qt;
        if (edge) mask_scores(z, a0, a1);
        float mx = -INFINITY;
#pragma unroll
        for (int k = 0; k < 16; ++k) mx = fmaxf(mx, z[k]);
        if (__any(mx * c > m + kLazy)) {
            float t = mx * c;
            t = fmaxf(t, __shfl_xor(t, 16, 64));
            t = fmaxf(t, __shfl_xor(t, 32, 64));
            const float mn = fmaxf(m, t);
            const float f = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= f;
#pragma unroll
            for (int d = 0; d < ND; ++d) acc[d] *= f;
        }
        const float b = score_offset(log_r, m);
#pragma unroll
        for (int k = 0; k < 16; ++k) z[k] = __builtin_amdgcn_exp2f(fmaf(z[k], c, b));
        float sum = 0.0f;
        f16x8 pf[2];
        uint32_t pw[8];
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            sum += z[i];
            sum += z[i + 1];
            pw[i / 2] = pack_f16(z[i], z[i + 1]);
        }
        l = fmaf(sum, inv_r, l);
        if (bad_scales(ks, vs)) l = bad_sum(l, lo, hi, j0);
        pf[0] = __builtin_bit_cast(f16x8, u32x4v{pw[0], pw[1], pw[2], pw[3]});
        pf[1] = __builtin_bit_cast(f16x8, u32x4v{pw[4], pw[5], pw[6], pw[7]});
        if (j0 + kKvBlock > len) {
#pragma unroll
            for (int d = 0; d < ND; ++d) vf[d] = keep_tokens(vf[d], len - j0 - 16 * qt);
        }
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            const f16x8 v0 = cvt8<KT>(vf[d].x, vf[d].y);
            const f16x8 v1 = cvt8<KT>(vf[d].z, vf[d].w);
            acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pf[0], acc[d], 0, 0, 0);
            acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pf[1], acc[d], 0, 0, 0);
        }
        load_v(next);
    }

    // Blocks first, first + stride, ... below nb of the request's blocks from b0
    // on.
    __device__ __forceinline__ void walk(const KvAttnArgs& a, const KvRequest& q, int64_t tile, int64_t r,
                                         int h, int b0, int nb, int first, int stride) {
        const int lane = threadIdx.x & 63;
        uint4 raw[2 * NK];
        int tok;
        fetch(a, q, tile, h, raw, tok);
        clear();
        // Lane i holds the number and scales of the wave's i-th of the current
        // 64 blocks; absent blocks are stepped over.
        KvBlockRef refs;
        const int cnt = first < nb ? (nb - first + stride - 1) / stride : 0;
        auto next = [&](int i, KvBlockRef& b) {
            for (; i < cnt; ++i) {
                if ((i & 63) == 0) {
                    refs.blk = -1;
                    refs.ks = refs.vs = 0.0f;
                    if (i + lane < cnt) refs = kv_block_ref(a, r, b0 + first + (i + lane) * stride, h);
                    // Wait for them here, not wherever the paths meet again (which
                    // would wait for every code on its way as well).
                    asm volatile("" : "+v"(refs.blk), "+v"(refs.ks), "+v"(refs.vs));
                }
                b = kv_lane_ref(refs, i & 63);
                if (b.blk >= 0) break;
            }
            return i;
        };
        auto codes = [&](int blk) {
            return a.c.codes + ((int64_t)blk * a.c.Hk + h) * 2 * kKvBlock * D;
        };
        KvBlockRef cur, nxt;
        int i = next(0, cur);
        if (i < cnt) {
            load_k(codes(cur.blk));
            load_v(codes(cur.blk));
        }
        start(a, q, raw, tok);
        while (i < cnt) {
            nxt = cur;
            const int in = next(i + 1, nxt);
            // Past the last block the loads repeat it (cached, and in bounds).
            const int to = in < cnt ? nxt.blk : cur.blk;
            block(cur.ks, cur.vs, (b0 + first + i * stride) * kKvBlock, q.len, codes(to));
            i = in;
            cur = nxt;
        }
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
    }
};

// LDS of W waves: sums [wave][D / 16][64 lanes] float4, then m, l and vref
// [wave][16 rows].
template <int D, int W>
constexpr int kXchgFloats = W * kRows * (D + 3);

// Joins the waves' sums; each wave's 16-dim tiles of a row go to o, or to `part`
// before the division by l.
template <int KT, int D, int W>
__device__ __forceinline__ void join_waves(const KvAttnArgs& a, const KvRequest& q, int64_t tile, int h,
                                           const RowsState<KT, D>& st, float* xs, float* part) {
    constexpr int ND = D / 16;
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, col = lane & 15;
    float* xm = xs + W * kRows * D;
    float* xl = xm + W * kRows;
    float* xu = xl + W * kRows;
    __syncthreads();  // an earlier pair's reads are over
#pragma unroll
    for (int d = 0; d < ND; ++d)
        reinterpret_cast<f32x4*>(xs)[(wv * ND + d) * 64 + lane] = st.acc[d];
    if (lane < kRows) {
        xm[wv * kRows + col] = st.m;
        xl[wv * kRows + col] = st.l;
        xu[wv * kRows + col] = st.vref;
    }
    __syncthreads();
    float f[W], mx = -INFINITY, unit = 0.0f, l = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        mx = fmaxf(mx, xm[w * kRows + col]);
        unit = fmaxf(unit, xu[w * kRows + col]);
    }
    const float base = mx == -INFINITY ? 0.0f : mx;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        f[w] = __builtin_amdgcn_exp2f(xm[w * kRows + col] - base);
        l = fmaf(xl[w * kRows + col], f[w], l);
        f[w] *= unit_ratio(xu[w * kRows + col], unit);
    }
    const int64_t i = tile * kRows + col;
    const bool real = i < (int64_t)q.n * a.G;
    const int tok = real ? (int)i / a.G : 0, head = h * a.G + (real ? (int)i - tok * a.G : 0);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int d0 = 0; d0 < ND; d0 += W) {
        const int d = d0 + wv;
        if (d >= ND) break;
        f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < W; ++w)
            s += reinterpret_cast<const f32x4*>(xs)[(w * ND + d) * 64 + lane] * f[w];
        const int at = d * 16 + 4 * (lane >> 4);
        if (part) {
            *reinterpret_cast<f32x4*>(part + col * D + at) = s;
        } else if (real) {
            *reinterpret_cast<uint2*>(a.o + (q.row0 + tok) * a.ld_o + (int64_t)head * D + at) =
                pack_bf16(s[0] * inv * unit, s[1] * inv * unit, s[2] * inv * unit, s[3] * inv * unit);
        }
    }
    if (part && threadIdx.x < kRows) {
        part[kRows * D + col] = mx;
        part[kRows * (D + 1) + col] = l;
        part[kRows * (D + 2) + col] = unit;
    }
}

template <int KT, int D, int W, bool SHARES>
__global__ __launch_bounds__(W * 64) __attribute__((amdgpu_waves_per_eu(D == 256 ? 1 : 2)))
void k_attention_rows(KvAttnArgs a, int64_t* __restrict__ plan, float* __restrict__ parts) {
    __shared__ __attribute__((aligned(16))) float xs[kXchgFloats<D, W>];
    const int wv = threadIdx.x >> 6;
    RowsState<KT, D> st;
    if constexpr (!SHARES) {
        int64_t r, tile;
        const int h = (int)(blockIdx.x % a.c.Hk);
        const KvRequest q = kv_slot_request<kRows>(a, blockIdx.x / a.c.Hk, r, tile);
        if (tile < 0 || tile * kRows >= (int64_t)q.n * a.G) return;
        st.walk(a, q, tile, r, h, q.block0, q.block1 - q.block0, wv, W);
        join_waves<KT, D, W>(a, q, tile, h, st, xs, nullptr);
    } else {
        __shared__ int64_t found[2 * W + 2];
        KvWalk<kRows, W> wk;
        if (!wk.start(a, kMinShare, plan, found)) return;
        while (wk.next(a)) {
            st.walk(a, wk.q, wk.tile, wk.r, wk.h, wk.q.block0 + wk.b0, wk.nb, wv, W);
            join_waves<KT, D, W>(a, wk.q, wk.tile, wk.h, st, xs,
                                 wk.whole() ? nullptr : parts + wk.part() * kv_part_floats<D, kRows>);
        }
    }
}

template <int KT, int D, int W>
void whole(const KvAttnArgs& a, hipStream_t s) {
    const int64_t grid = kv_slots(a.c.T, a.c.R, a.G, kRows) * a.c.Hk;
    k_attention_rows<KT, D, W, false><<<(unsigned)grid, W * 64, 0, s>>>(a, nullptr, nullptr);
}

template <int KT, int D>
hipError_t rows_of(const KvAttnArgs& a, int waves, hipStream_t s) {
    if (waves == 0) {
        int64_t* plan = reinterpret_cast<int64_t*>(a.ws);
        float* parts = reinterpret_cast<float*>(reinterpret_cast<char*>(a.ws) + kv_plan_bytes(a.c.R));
        k_attention_rows<KT, D, 4, true><<<kRowsShares, 256, 0, s>>>(a, plan, parts);
    } else if (waves == 1) {
        whole<KT, D, 1>(a, s);
    } else if (waves == 2) {
        whole<KT, D, 2>(a, s);
    } else if (waves == 4 || D == 256) {
        whole<KT, D, 4>(a, s);
    } else {
        if constexpr (D < 256) whole<KT, D, 8>(a, s);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_rows(readme_kv_type kt, const KvAttnArgs& a, int waves, hipStream_t s) {
    const bool i8 = kt == README_KV_I8;
    switch (a.c.D) {
        case 64: return i8 ? rows_of<README_KV_I8, 64>(a, waves, s) : rows_of<README_KV_E4M3, 64>(a, waves, s);
        case 128: return i8 ? rows_of<README_KV_I8, 128>(a, waves, s) : rows_of<README_KV_E4M3, 128>(a, waves, s);
        case 256: return i8 ? rows_of<README_KV_I8, 256>(a, waves, s) : rows_of<README_KV_E4M3, 256>(a, waves, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace readme
