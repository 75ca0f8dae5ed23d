// Attention over the 8-bit cache for the rows of draft trees (attention_kv.hpp has
// the mathematics): 32 query rows a wave.
//
// The waves of a workgroup take the blocks of a (request, 32 rows, key head) pair in
// turn, each block's codes straight from memory to the registers of the matrix
// operands, with no LDS and no barrier:
//     S^T = K Q^T   32x32x16 MFMA; a lane gets 16 scores of one row for each half of
//                   the block, of the 16 tokens whose codes it loads for V, so P
//                   stays in its registers;
//     O^T += V^T P^T.
// The codes' conversion to fp16 is paid once for 32 rows.  The waves' sums meet in LDS
// at the end of a pair.
//
// Bound by instructions: a block asks a wave (heads of 128) for 32 products of 32 clocks
// and, for them, 128 (e4m3) or 256 (int8) conversions and about 160 steps of softmax of 4
// clocks and more.  16 requests of 32 rows over 1000 to 4096 tokens (four query heads to a
// key head, e4m3): 43 us, of the SIMDs' busy cycles 59% vector ALU and 31% products;
// the call reads and writes 93 MB, 18 us as a copy, its products are 16 us at a large
// product's rate; launch, first loads and the join of the waves are 9 of the 43.
// Two waves a SIMD: 235 to 256 registers, one spilled in three of the e4m3 forms.
// What did not help, the same call at 45 us: 64 rows a wave, with Q in registers or in
// LDS, halves the conversions and spills, 90 to 130; a wave's priority raised over its
// products, and P's sums by dot products, no difference.
#include <math.h>

#include "attention_kv.hpp"

namespace readme {

namespace {

constexpr int kRows = kTreeTile;
constexpr int kMinShare = 16;

// One wave's running result over the blocks it takes, for 32 rows.
template <int KT, int D>
struct TreeState {
    static constexpr int NQ = D / 16;
    static constexpr int ND = D / 32;  // 32-dim tiles, and 16-byte pieces of half a block
    f16x8 qf[NQ];
    f32x16 acc[ND];
    uint4 kf[2][ND], vf[2][ND];
    float m, l, cq, vref, log_vref;
    int max_lo;  // over the rows: from there to the first own row blocks are seen whole
    TreeRow tr;

    __device__ __forceinline__ void fetch(const KvAttnArgs& a, const KvRequest& q, int64_t tile, int h,
                                          uint4 (&raw)[NQ], int& pos) {
        const int lane = threadIdx.x & 63, col = lane & 31, hf = lane >> 5;
        const int64_t i = tile * kRows + col;
        const bool real = i < (int64_t)q.n * a.G;
        const int t = real ? (int)i / a.G : 0;  // i < n G <= 2^27
        const int head = h * a.G + (real ? (int)i - t * a.G : 0);
        const uint16_t* row = a.q + (q.row0 + t) * a.ld_q + (int64_t)head * D;
#pragma unroll
        for (int s = 0; s < NQ; ++s) {
            raw[s] = make_uint4(0u, 0u, 0u, 0u);
            if (real) raw[s] = *reinterpret_cast<const uint4*>(row + (s >> 1) * 32 + hf * 16 + (s & 1) * 8);
        }
        tr.tok = real ? t : -1;
        pos = TreeRow::position(a, q, tr.tok);
    }

    __device__ __forceinline__ void start(const KvAttnArgs& a, const KvRequest& q, const uint4 (&raw)[NQ],
                                          int pos) {
        tr.set(a, q, tr.tok, pos);
        float big = 0.0f;
#pragma unroll
        for (int s = 0; s < NQ; ++s) {
            const uint32_t v[4] = {raw[s].x, raw[s].y, raw[s].z, raw[s].w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                big = fmaxf(big, fmaxf(fabsf(bf16_lo(v[e])), fabsf(bf16_hi(v[e]))));
        }
        big = fmaxf(big, __shfl_xor(big, 32, 64));
        float up, down;
        row_power(big, up, down);
        cq = a.score * down;
#pragma unroll
        for (int s = 0; s < NQ; ++s) {
            const uint32_t v[4] = {raw[s].x, raw[s].y, raw[s].z, raw[s].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                qf[s][2 * e] = (_Float16)(bf16_lo(v[e]) * up);
                qf[s][2 * e + 1] = (_Float16)(bf16_hi(v[e]) * up);
            }
        }
        max_lo = tr.tok >= 0 ? tr.lo : 0;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) max_lo = max(max_lo, __shfl_xor(max_lo, off, 64));
        max_lo = __builtin_amdgcn_readfirstlane(max_lo);
        m = -INFINITY;
        l = 0.0f;
        vref = log_vref = 0.0f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[d][k] = 0.0f;
    }

    // Key row m of an operand is token 16 (m / 4 % 2) + 4 (m / 8) + m % 4 of the half,
    // so that result row i of a lane is token 16 (lane / 32) + i.
    __device__ __forceinline__ void load_k(const uint8_t* codes) {
        const int lane = threadIdx.x & 63, row = lane & 31, hf = lane >> 5;
        const int tok = 16 * ((row >> 2) & 1) + 4 * (row >> 3) + (row & 3);
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int u = 0; u < ND; ++u)
                kf[g][u] = *reinterpret_cast<const uint4*>(codes + ((g * (D / 16) + 2 * u + hf) * 32 + tok) * 16);
    }
    __device__ __forceinline__ void load_v(const uint8_t* codes) {
        const int lane = threadIdx.x & 63, row = lane & 31, hf = lane >> 5;
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int d = 0; d < ND; ++d)
                vf[g][d] = *reinterpret_cast<const uint4*>(codes + kKvBlock * D + (g * D + d * 32 + row) * 32 +
                                                           hf * 16);
    }

    // The block held in kf and vf, its token 0 at position j0; `next` is the block
    // whose codes take its place.
    __device__ __forceinline__ void block(const KvAttnArgs& a, const KvRequest& q, float ks, float vs, int j0,
                                          const uint8_t* next) {
        const int hf = (threadIdx.x & 63) >> 5;
        f32x16 s[2];
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int k = 0; k < 16; ++k) s[g][k] = 0.0f;
#pragma unroll
        for (int u = 0; u < ND; ++u)
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const f16x8 k0 = cvt8<KT>(kf[g][u].x, kf[g][u].y);
                const f16x8 k1 = cvt8<KT>(kf[g][u].z, kf[g][u].w);
                s[g] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k0, qf[2 * u], s[g], 0, 0, 0);
                s[g] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k1, qf[2 * u + 1], s[g], 0, 0, 0);
            }
        load_k(next);

        const bool edge = j0 + kKvBlock > q.len - q.n || j0 < max_lo;
        uint64_t seen = ~0ull;
        if (edge) seen = tr.seen(a, q, j0);
        const bool sees = seen != 0;
        value_unit(vs, sees, vref, log_vref, acc, [](float x) { return fmaxf(x, __shfl_xor(x, 32, 64)); });
        float log_r, inv_r;
        value_ratio(vs, log_vref, log_r, inv_r);
        const float c = score_factor(cq, ks);
        // score (g, k) is token j0 + 32 g + 16 hf + k
        if (edge) {
            mask_bits(s[0], (uint32_t)(seen >> (16 * hf)));
            mask_bits(s[1], (uint32_t)(seen >> (16 * hf + 32)));
        }
        float mx = -INFINITY;
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int k = 0; k < 16; ++k) mx = fmaxf(mx, s[g][k]);
        if (__any(mx * c > m + kLazy)) {
            float t = mx * c;
            t = fmaxf(t, __shfl_xor(t, 32, 64));
            const float mn = fmaxf(m, t);
            const float f = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= f;
#pragma unroll
            for (int d = 0; d < ND; ++d) acc[d] *= f;
        }
        const float b = score_offset(log_r, m);
        if (j0 + kKvBlock > q.len) {
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int d = 0; d < ND; ++d) vf[g][d] = keep_tokens(vf[g][d], q.len - j0 - 32 * g - 16 * hf);
        }
        float sum = 0.0f;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            f16x8 pf[2];
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                u32x4v pw;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float p0 = __builtin_amdgcn_exp2f(fmaf(s[g][8 * st + 2 * k], c, b));
                    const float p1 = __builtin_amdgcn_exp2f(fmaf(s[g][8 * st + 2 * k + 1], c, b));
                    sum += p0;
                    sum += p1;
                    pw[k] = pack_f16(p0, p1);
                }
                pf[st] = __builtin_bit_cast(f16x8, pw);
            }
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                const f16x8 v0 = cvt8<KT>(vf[g][d].x, vf[g][d].y);
                const f16x8 v1 = cvt8<KT>(vf[g][d].z, vf[g][d].w);
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v0, pf[0], acc[d], 0, 0, 0);
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v1, pf[1], acc[d], 0, 0, 0);
            }
        }
        load_v(next);
        l = fmaf(sum, inv_r, l);
        if (bad_scales(ks, vs) && sees) l = __builtin_nanf("");
    }

    // Blocks first, first + stride, ... below nb of the request's blocks from b0 on.
    template <int W>
    __device__ __forceinline__ void walk(const KvAttnArgs& a, const KvRequest& q, int64_t tile, int64_t r,
                                         int h, int b0, int nb) {
        const int lane = threadIdx.x & 63;
        const int first = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        uint4 raw[NQ];
        int pos;
        fetch(a, q, tile, h, raw, pos);
        // Lane i holds the number and scales of the wave's i-th of the current 64
        // blocks; absent blocks are stepped over.
        KvBlockRef refs;
        const int cnt = first < nb ? (nb - first + W - 1) / W : 0;
        auto number = [&](int i) {
            refs.blk = -1;
            if (i + lane < cnt)
                refs.blk = (int)kv_block_of(a.c.table, a.c.max_blocks, a.c.n_blocks, r, b0 + first + (i + lane) * W);
            // Wait for them here, not wherever the paths meet again (which would
            // wait for every code on its way as well).
            asm volatile("" : "+v"(refs.blk));
        };
        auto next = [&](int i, KvBlockRef& b) {
            for (; i < cnt; ++i) {
                if ((i & 63) == 0 && i > 0) {
                    number(i);
                    kv_set_scales(refs, kv_block_scales(a, refs.blk, h));
                    asm volatile("" : "+v"(refs.ks), "+v"(refs.vs));
                }
                b = kv_lane_ref(refs, i & 63);
                if (b.blk >= 0) break;
            }
            return i;
        };
        auto codes = [&](int blk) {
            return a.c.codes + ((int64_t)blk * a.c.Hk + h) * 2 * kKvBlock * D;
        };
        // The first codes follow their blocks' numbers at once, the scales on their
        // way beside them: one round to memory less before the first score.
        number(0);
        const float2 scales = kv_block_scales(a, refs.blk, h);
        refs.ks = refs.vs = 0.0f;
        KvBlockRef cur, nxt;
        int i = next(0, cur);
        if (i < cnt) {
            load_k(codes(cur.blk));
            load_v(codes(cur.blk));
        }
        start(a, q, raw, pos);
        if (i < 64) {
            kv_set_scales(refs, scales);
            asm volatile("" : "+v"(refs.ks), "+v"(refs.vs));
            cur = kv_lane_ref(refs, i);
        }
        while (i < cnt) {
            nxt = cur;
            const int in = next(i + 1, nxt);
            // Past the last block the loads repeat it (cached, and in bounds).
            const int to = in < cnt ? nxt.blk : cur.blk;
            block(a, q, cur.ks, cur.vs, (b0 + first + i * W) * kKvBlock, codes(to));
            i = in;
            cur = nxt;
        }
        l += __shfl_xor(l, 32, 64);
    }
};

// LDS of W waves for a 32-dim tile of the sums [wave][4][64 lanes] float4, and m, l
// and vref [wave][rows].
template <int W>
constexpr int kXchgFloats = W * kRows * (32 + 3);

// Joins the waves' sums, 32 dims at a time; each wave's share of them goes to o, or to
// `part` before the division by l.
template <int D, int W, class State>
__device__ __forceinline__ void join_waves(const KvAttnArgs& a, const KvRequest& q, int64_t tile, int h,
                                           const State& st, float* xs, float* part) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, col = lane & 31;
    float* xm = xs + W * kRows * 32;
    float* xl = xm + W * kRows;
    float* xu = xl + W * kRows;
    __syncthreads();  // an earlier pair's reads are over
    if (lane < 32) {
        xm[wv * kRows + lane] = st.m;
        xl[wv * kRows + lane] = st.l;
        xu[wv * kRows + lane] = st.vref;
    }
    const int64_t i = tile * kRows + col;
    const bool real = i < (int64_t)q.n * a.G;
    const int tok = real ? (int)i / a.G : 0, head = h * a.G + (real ? (int)i - tok * a.G : 0);
    uint16_t* row = a.o + (q.row0 + tok) * a.ld_o + (int64_t)head * D;
    float f[W], mx = -INFINITY, unit = 0.0f, l = 0.0f, inv = 0.0f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
        if (d > 0) __syncthreads();  // the last tile's reads are over
#pragma unroll
        for (int p = 0; p < 4; ++p)
            reinterpret_cast<f32x4*>(xs)[(wv * 4 + p) * 64 + lane] =
                f32x4{st.acc[d][4 * p], st.acc[d][4 * p + 1], st.acc[d][4 * p + 2], st.acc[d][4 * p + 3]};
        __syncthreads();
        if (d == 0) {
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
            inv = l == 0.0f ? 0.0f : 1.0f / l;
        }
#pragma unroll
        for (int p0 = 0; p0 < 4; p0 += W) {
            const int p = p0 + wv;
            if (p >= 4) break;
            f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < W; ++w) s += reinterpret_cast<const f32x4*>(xs)[(w * 4 + p) * 64 + lane] * f[w];
            const int at = d * 32 + 8 * p + 4 * (lane >> 5);
            if (part)
                *reinterpret_cast<f32x4*>(part + col * D + at) = s;
            else if (real)
                *reinterpret_cast<uint2*>(row + at) =
                    pack_bf16(s[0] * inv * unit, s[1] * inv * unit, s[2] * inv * unit, s[3] * inv * unit);
        }
    }
    if (part && threadIdx.x < 32) {
        part[kRows * D + col] = mx;
        part[kRows * (D + 1) + col] = l;
        part[kRows * (D + 2) + col] = unit;
    }
}

// A walk's place is the same for all lanes: in scalar registers it takes none of the
// vector registers that the blocks need.
template <class Walk>
__device__ __forceinline__ void to_scalars(Walk& w) {
    auto s32 = [](int& x) { x = __builtin_amdgcn_readfirstlane(x); };
    auto s64 = [](int64_t& x) { x = wave_uniform(x); };
    s64(w.w), s64(w.w1), s64(w.base), s64(w.r), s64(w.tile), s64(w.q.row0), s64(w.p.weight);
    s32(w.h), s32(w.b0), s32(w.nb), s32(w.q.n), s32(w.q.len), s32(w.q.block0), s32(w.q.block1);
    s32(w.p.tiles), s32(w.p.blocks);
}

template <int KT, int D, int W, bool SHARES>
__global__ __launch_bounds__(W * 64) __attribute__((amdgpu_waves_per_eu(2, 2)))
void k_attention_tree(KvAttnArgs a, int64_t* __restrict__ plan, float* __restrict__ parts, int64_t run) {
    __shared__ __attribute__((aligned(16))) float xs[kXchgFloats<W>];
    TreeState<KT, D> st;
    if constexpr (!SHARES) {
        // Runs of `run` row tiles, about a request's, go to one of the eight dies: they
        // read the same codes, which then come from its L2.
        const int64_t S = kv_slots(a.c.T, a.c.R, a.G, kRows), j = blockIdx.x >> 3;
        const int64_t at = ((j / run) * 8 + (blockIdx.x & 7)) * run + j % run;
        if (at >= S * a.c.Hk) return;
        const int h = (int)(at / S);
        int64_t r, tile;
        const KvRequest q = kv_slot_request<kRows>(a, at - h * S, r, tile);
        if (tile < 0 || tile * kRows >= (int64_t)q.n * a.G) return;
        st.template walk<W>(a, q, tile, r, h, q.block0, q.block1 - q.block0);
        join_waves<D, W>(a, q, tile, h, st, xs, nullptr);
    } else {
        __shared__ int64_t found[2 * W + 2];
        KvWalk<kRows, W> wk;
        if (!wk.start(a, kMinShare, plan, found)) return;
        while (wk.next(a)) {
            to_scalars(wk);
            st.template walk<W>(a, wk.q, wk.tile, wk.r, wk.h, wk.q.block0 + wk.b0, wk.nb);
            join_waves<D, W>(a, wk.q, wk.tile, wk.h, st, xs,
                             wk.whole() ? nullptr : parts + wk.part() * kv_part_floats<D, kRows>);
        }
    }
}

template <int KT, int D, int W>
void whole(const KvAttnArgs& a, hipStream_t s) {
    const int64_t S = kv_slots(a.c.T, a.c.R, a.G, kRows);
    int64_t run = S / a.c.R;  // at least 1
    run = run < 16 ? run : 16;
    const int64_t grid = ceil_div(S * a.c.Hk, 8 * run) * 8 * run;
    k_attention_tree<KT, D, W, false><<<(unsigned)grid, W * 64, 0, s>>>(a, nullptr, nullptr, run);
}

template <int KT, int D>
hipError_t tree_of(const KvAttnArgs& a, int waves, hipStream_t s) {
    if (waves == 0) {
        int64_t* plan = reinterpret_cast<int64_t*>(a.ws);
        float* parts = reinterpret_cast<float*>(reinterpret_cast<char*>(a.ws) + kv_plan_bytes(a.c.R));
        k_attention_tree<KT, D, 4, true><<<kTreeShares, 256, 0, s>>>(a, plan, parts, 0);
    } else if (waves == 1) {
        whole<KT, D, 1>(a, s);
    } else if (waves == 2) {
        whole<KT, D, 2>(a, s);
    } else if (waves == 4) {
        whole<KT, D, 4>(a, s);
    } else {
        whole<KT, D, 8>(a, s);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_tree(readme_kv_type kt, const KvAttnArgs& a, int waves, hipStream_t s) {
    const bool i8 = kt == README_KV_I8;
    switch (a.c.D) {
        case 64: return i8 ? tree_of<README_KV_I8, 64>(a, waves, s) : tree_of<README_KV_E4M3, 64>(a, waves, s);
        case 128: return i8 ? tree_of<README_KV_I8, 128>(a, waves, s) : tree_of<README_KV_E4M3, 128>(a, waves, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace readme
