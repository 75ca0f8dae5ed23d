// Attention over the 8-bit cache for many query rows: prompts and pieces of
// prompts (attention_kv.hpp has the mathematics).
//
// A workgroup holds 128 query rows of one key head (a row is a token and one of
// its G query heads, so G heads share each key), four waves of 32, and walks
// over the blocks of 64 tokens.  The four waves fetch a block's codes together,
// turn them into fp16 once and write them to one of two LDS buffers in the order
// of the matrix operands, the next block's codes in flight meanwhile; one barrier
// a block.  Per wave and 32 tokens, 32x32x16 MFMA:
//     S^T = K Q^T   a lane gets 16 scores of one row, of the 16 tokens that its
//                   V operand holds, so P stays in its registers and a row's
//                   maximum needs one exchange (lane ^ 32), only when it grows;
//     O^T += V^T P^T   a lane's sums are all of one row, so rescaling is one
//                   multiply by a factor of its own.
// Measured (heads of 128, 32 on 8 key heads): 8 x 2048 rows on 2048 keys each,
// not causal, 603 us, 911 TFLOP/s; 4 causal prompts of 2048, int8 166 to 171 us by
// the card (804 to 828; 176 for a pass alone), e4m3 151; the matrix cores busy 40% of
// the cycles and the LDS 31%, with no bank conflicts.  What the rest waits for is
// spread out: of the first's time (595 us in that run) the operand reads between the
// products are worth 208, the exponentials 20, the staging 44.  Not faster: a half
// block's scores ahead of its softmax (650), 64 rows a wave at one wave a SIMD (730)
// or, for heads of 64, at two (116 us where this takes 112, 151 for 82 where shares
// are dealt), three waves a SIMD for heads of 64 (the same).
#include <math.h>

#include "attention_kv.hpp"

namespace readme {

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr int kMinShare = 8;
constexpr int kSchedMfma = 0x8, kSchedRead = 0x100;  // __builtin_amdgcn_sched_group_barrier

template <int KT, int D>
struct TileState {
    static constexpr int NQ = D / 16;  // steps of Q K^T, and 32-dim tiles x 2
    static constexpr int ND = D / 32;
    f16x8 qf[NQ];
    f32x16 acc[ND];
    float m, l, cq, vref, log_vref;
    int lo, hi;                  // keys this lane's row sees
    int min_hi, max_hi, min_lo, max_lo;  // over the wave's rows
    bool real;                   // the lane's row exists
    int64_t out;                 // its place in o

    __device__ __forceinline__ void start(const KvAttnArgs& a, const KvRequest& q, int64_t tile, int h) {
        const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, col = lane & 31, hf = lane >> 5;
        const int64_t i = tile * kTilesTile + wv * 32 + col;
        real = i < (int64_t)q.n * a.G;
        const int64_t tok = real ? i / a.G : 0;
        const int64_t head = (int64_t)h * a.G + (real ? i - tok * a.G : 0);
        const uint16_t* row = a.q + (q.row0 + tok) * a.ld_q + head * D;
        out = (q.row0 + tok) * a.ld_o + head * D;
        uint4 raw[NQ];
        float big = 0.0f;
#pragma unroll
        for (int s = 0; s < NQ; ++s) {
            raw[s] = make_uint4(0u, 0u, 0u, 0u);
            if (real) raw[s] = *reinterpret_cast<const uint4*>(row + (s >> 1) * 32 + hf * 16 + (s & 1) * 8);
        }
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
        row_keys(a, q.len, (int64_t)q.len - q.n + tok, lo, hi);
        min_hi = real ? hi : 0x7fffffff;
        max_hi = real ? hi : 0;
        min_lo = real ? lo : 0x7fffffff;
        max_lo = real ? lo : 0;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            min_hi = min(min_hi, __shfl_xor(min_hi, off, 64));
            max_hi = max(max_hi, __shfl_xor(max_hi, off, 64));
            min_lo = min(min_lo, __shfl_xor(min_lo, off, 64));
            max_lo = max(max_lo, __shfl_xor(max_lo, off, 64));
        }
        // Uniform over the wave (the two halves hold the same rows)
        min_hi = __builtin_amdgcn_readfirstlane(min_hi);
        max_hi = __builtin_amdgcn_readfirstlane(max_hi);
        min_lo = __builtin_amdgcn_readfirstlane(min_lo);
        max_lo = __builtin_amdgcn_readfirstlane(max_lo);
        m = -INFINITY;
        l = 0.0f;
        vref = log_vref = 0.0f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[d][k] = 0.0f;
    }

    // The block whose token 0 is at position j0, K operands at kl, V at vl.
    __device__ __forceinline__ void block(const uint8_t* kl, const uint8_t* vl, float ks, float vs, int j0) {
        if (j0 >= max_hi || j0 + kKvBlock <= min_lo) return;
        const int lane = threadIdx.x & 63, hf = lane >> 5;
        // Operands are read kAhead steps before their product, so that an LDS
        // round trip hides behind other products (4 and 6: the same time, and
        // registers spilled where shares are dealt).
        constexpr int kAhead = 2;
        auto k_at = [&](int i) {  // step i: token half i % 2, dims i / 2
            return *reinterpret_cast<const f16x8*>(kl + (((i & 1) * NQ + (i >> 1)) * 64 + lane) * 16);
        };
        auto v_at = [&](int i) {
            return *reinterpret_cast<const f16x8*>(vl + (i * 64 + lane) * 16);
        };
        f32x16 s[2];
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int k = 0; k < 16; ++k) s[g][k] = 0.0f;
        {
            f16x8 f[2 * NQ];
#pragma unroll
            for (int i = 0; i < 2 * NQ; ++i) f[i] = k_at(i);
#pragma unroll
            for (int i = 0; i < 2 * NQ; ++i)
                s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[i], qf[i >> 1], s[i & 1], 0, 0, 0);
            __builtin_amdgcn_sched_group_barrier(kSchedRead, kAhead, 0);
#pragma unroll
            for (int i = 0; i < 2 * NQ - kAhead; ++i) {
                __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kSchedRead, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(kSchedMfma, kAhead, 0);
        }
        f16x8 vf[4 * ND];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) vf[i] = v_at(i);
        const bool edge = j0 + kKvBlock > min_hi || j0 < max_lo;
        value_unit(vs, !edge || sees_block(lo, hi, j0), vref, log_vref, acc,
                   [](float x) { return fmaxf(x, __shfl_xor(x, 32, 64)); });
        float log_r, inv_r;
        value_ratio(vs, log_vref, log_r, inv_r);
        const float c = score_factor(cq, ks);
        // score (g, k) is token j0 + 32 g + 16 hf + k
        const int a0 = lo - j0 - 16 * hf, a1 = hi - j0 - 16 * hf;
        if (edge) {
            mask_scores(s[0], a0, a1);
            mask_scores(s[1], a0 - 32, a1 - 32);
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
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int k = 0; k < 16; ++k) s[g][k] = __builtin_amdgcn_exp2f(fmaf(s[g][k], c, b));
        float sum = 0.0f;
        f16x8 pf[4];
#pragma unroll
        for (int st = 0; st < 4; ++st) {
            u32x4v pw;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float p0 = s[st >> 1][8 * (st & 1) + 2 * k], p1 = s[st >> 1][8 * (st & 1) + 2 * k + 1];
                sum += p0;
                sum += p1;
                pw[k] = pack_f16(p0, p1);
            }
            pf[st] = __builtin_bit_cast(f16x8, pw);
        }
#pragma unroll
        for (int i = kAhead; i < 4 * ND; ++i) vf[i] = v_at(i);
#pragma unroll
        for (int i = 0; i < 4 * ND; ++i)
            acc[i % ND] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[i], pf[i / ND], acc[i % ND], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4 * ND - kAhead; ++i) {
            __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kSchedRead, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kSchedMfma, kAhead, 0);
        l = fmaf(sum, inv_r, l);
        if (bad_scales(ks, vs)) l = bad_sum(l, lo, hi, j0);
    }

    __device__ __forceinline__ void finish() { l += __shfl_xor(l, 32, 64); }

    __device__ __forceinline__ void store(const KvAttnArgs& a) const {
        if (!real) return;
        const int hf = (threadIdx.x & 63) >> 5;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        uint16_t* row = a.o + out + 4 * hf;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<uint2*>(row + d * 32 + 8 * g) =
                    pack_bf16(acc[d][4 * g] * inv * vref, acc[d][4 * g + 1] * inv * vref,
                              acc[d][4 * g + 2] * inv * vref, acc[d][4 * g + 3] * inv * vref);
    }
    __device__ __forceinline__ void store_part(float* part) const {
        const int lane = threadIdx.x & 63, i = (threadIdx.x >> 6) * 32 + (lane & 31), hf = lane >> 5;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4*>(part + i * D + d * 32 + 8 * g + 4 * hf) =
                    f32x4{acc[d][4 * g], acc[d][4 * g + 1], acc[d][4 * g + 2], acc[d][4 * g + 3]};
        if (hf == 0) {
            part[kTilesTile * D + i] = m;
            part[kTilesTile * (D + 1) + i] = l;
            part[kTilesTile * (D + 2) + i] = vref;
        }
    }
};

// A block's codes on their way from memory to LDS operands.  Thread piece i is
// lane `lane` of K operand pair (g, u, u + 1) and of V operand pair (g, d):
// sixteen dims of key row m = lane % 32, which is token 16 (m / 4 % 2) + 4 (m / 8)
// + m % 4 of the half, so that result row i of a lane is token 16 (lane / 32) + i;
// sixteen tokens of one dim.
template <int KT, int D>
struct Stage {
    static constexpr int N = D / 64;  // pieces a thread, of K and of V
    uint4 k[N], v[N];

    __device__ __forceinline__ void load(const uint8_t* codes) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int pi = threadIdx.x + i * kThreads, lane = pi & 63, f = pi >> 6;
            const int row = lane & 31, hf = lane >> 5;
            const int tok = 16 * ((row >> 2) & 1) + 4 * (row >> 3) + (row & 3);
            const int kg = f / (D / 32), u = f % (D / 32);
            k[i] = *reinterpret_cast<const uint4*>(codes + ((kg * (D / 16) + 2 * u + hf) * 32 + tok) * 16);
            const int vg = f / (D / 32), d = f % (D / 32);
            v[i] = *reinterpret_cast<const uint4*>(codes + kKvBlock * D + (vg * D + d * 32 + row) * 32 + hf * 16);
        }
    }
    // `keep` tokens of the block are in the cache.
    __device__ __forceinline__ void store(uint8_t* kl, uint8_t* vl, int keep) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int pi = threadIdx.x + i * kThreads, lane = pi & 63, f = pi >> 6, hf = lane >> 5;
            const int g = f / (D / 32), u = f % (D / 32);
            uint8_t* kd = kl + ((g * (D / 16) + 2 * u) * 64 + lane) * 16;
            *reinterpret_cast<f16x8*>(kd) = cvt8<KT>(k[i].x, k[i].y);
            *reinterpret_cast<f16x8*>(kd + 64 * 16) = cvt8<KT>(k[i].z, k[i].w);
            uint4 w = v[i];
            if (keep < kKvBlock) w = keep_tokens(w, keep - 32 * g - 16 * hf);
            uint8_t* vd = vl + ((g * 2 * (D / 32) + u) * 64 + lane) * 16;
            *reinterpret_cast<f16x8*>(vd) = cvt8<KT>(w.x, w.y);
            *reinterpret_cast<f16x8*>(vd + (D / 32) * 64 * 16) = cvt8<KT>(w.z, w.w);
        }
    }
};

// Blocks [b0, b0 + nb) of a request for the tile in `st`.
template <int KT, int D>
__device__ __forceinline__ void walk(const KvAttnArgs& a, const KvRequest& q, int64_t r, int h, int b0,
                                     int nb, uint8_t* lds, TileState<KT, D>& st) {
    constexpr int kBuf = kKvBlock * D * 2 * 2;  // K and V operands of a block
    const int lane = threadIdx.x & 63;
    Stage<KT, D> sg;
    auto codes_of = [&](int blk) {
        return a.c.codes + ((int64_t)blk * a.c.Hk + h) * 2 * kKvBlock * D;
    };
    // Lane i holds the number and scales of block i of the current 64; absent
    // blocks are stepped over, by all waves alike.
    KvBlockRef refs;
    auto refill = [&](int i) {
        refs.blk = -1;
        refs.ks = refs.vs = 0.0f;
        if (i + lane < nb) refs = kv_block_ref(a, r, b0 + i + lane, h);
        // Wait for them here, not wherever the paths meet again (which would wait
        // for every code on its way as well).
        asm volatile("" : "+v"(refs.blk), "+v"(refs.ks), "+v"(refs.vs));
    };
    auto next = [&](int i, KvBlockRef& b) {
        for (; i < nb; ++i) {
            if ((i & 63) == 0) refill(i);
            b = kv_lane_ref(refs, i & 63);
            if (b.blk >= 0) break;
        }
        return i;
    };
    KvBlockRef cur, nxt;
    int i = next(0, cur), buf = 0;
    if (i < nb) sg.load(codes_of(cur.blk));
    while (i < nb) {
        uint8_t* kl = lds + buf * kBuf;
        uint8_t* vl = kl + kKvBlock * D * 2;
        const int j0 = (b0 + i) * kKvBlock;
        sg.store(kl, vl, q.len - j0);
        const int in = next(i + 1, nxt);
        if (in < nb) sg.load(codes_of(nxt.blk));
        __syncthreads();
        st.block(kl, vl, cur.ks, cur.vs, j0);
        i = in;
        cur = nxt;
        buf ^= 1;
    }
    __syncthreads();  // the next walk writes the buffers from the first on
}

template <int KT, int D, bool SHARES>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(D == 256 ? 1 : 2)))
void k_attention_tiles(KvAttnArgs a, int64_t* __restrict__ plan, float* __restrict__ parts) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * kKvBlock * D * 2 * 2];
    TileState<KT, D> st;
    if constexpr (!SHARES) {
        // One pair a workgroup, head fastest.  The slots are taken as R columns of
        // equal length, from the bottom row up: with requests of like lengths that
        // is every request's last rows first, which see the most blocks, so that
        // long pairs do not start last.
        const int64_t S = kv_slots(a.c.T, a.c.R, a.G, kTilesTile), len = (S + a.c.R - 1) / a.c.R;
        const int64_t x = blockIdx.x / a.c.Hk;
        const int h = (int)(blockIdx.x % a.c.Hk);
        const int64_t slot = (x % a.c.R) * len + (len - 1 - x / a.c.R);
        if (slot >= S) return;
        int64_t r, tile;
        const KvRequest q = kv_slot_request<kTilesTile>(a, slot, r, tile);
        if (tile < 0 || tile * kTilesTile >= (int64_t)q.n * a.G) return;
        st.start(a, q, tile, h);
        // Blocks that any of the tile's rows sees: its first and last row's
        const int64_t t0 = tile * kTilesTile / a.G;
        int64_t t1 = (tile * kTilesTile + kTilesTile - 1) / a.G;
        t1 = t1 < q.n ? t1 : q.n - 1;
        int lo, hi, unused;
        row_keys(a, q.len, (int64_t)q.len - q.n + t0, lo, unused);
        row_keys(a, q.len, (int64_t)q.len - q.n + t1, unused, hi);
        const int b0 = lo / kKvBlock;
        int b1 = (hi + kKvBlock - 1) / kKvBlock;
        b1 = b1 < q.block1 ? b1 : q.block1;
        walk<KT, D>(a, q, r, h, b0, b1 - b0, lds, st);
        st.finish();
        st.store(a);
    } else {
        __shared__ int64_t found[2 * kWaves + 2];
        KvWalk<kTilesTile, kWaves> wk;
        if (!wk.start(a, kMinShare, plan, found)) return;
        while (wk.next(a)) {
            st.start(a, wk.q, wk.tile, wk.h);
            walk<KT, D>(a, wk.q, wk.r, wk.h, wk.q.block0 + wk.b0, wk.nb, lds, st);
            st.finish();
            if (wk.whole())
                st.store(a);
            else
                st.store_part(parts + wk.part() * kv_part_floats<D, kTilesTile>);
        }
    }
}

template <int KT, int D>
hipError_t tiles_of(const KvAttnArgs& a, bool shares, hipStream_t s) {
    int64_t* plan = reinterpret_cast<int64_t*>(a.ws);
    float* parts = reinterpret_cast<float*>(reinterpret_cast<char*>(a.ws) + kv_plan_bytes(a.c.R));
    if (shares) {
        k_attention_tiles<KT, D, true><<<kTilesShares, kThreads, 0, s>>>(a, plan, parts);
    } else {
        const int64_t grid = ceil_div(kv_slots(a.c.T, a.c.R, a.G, kTilesTile), a.c.R) * a.c.R * a.c.Hk;
        k_attention_tiles<KT, D, false><<<(unsigned)grid, kThreads, 0, s>>>(a, plan, parts);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_tiles(readme_kv_type kt, const KvAttnArgs& a, bool shares, hipStream_t s) {
    const bool i8 = kt == README_KV_I8;
    switch (a.c.D) {
        case 64: return i8 ? tiles_of<README_KV_I8, 64>(a, shares, s) : tiles_of<README_KV_E4M3, 64>(a, shares, s);
        case 128: return i8 ? tiles_of<README_KV_I8, 128>(a, shares, s) : tiles_of<README_KV_E4M3, 128>(a, shares, s);
        case 256: return i8 ? tiles_of<README_KV_I8, 256>(a, shares, s) : tiles_of<README_KV_E4M3, 256>(a, shares, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace readme
