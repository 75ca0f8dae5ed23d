// Shared by the two attention kernels over the 8-bit cache
// (attention_kv_rows.hpp: few query rows, attention_kv_tiles.hpp: many), each with
// rows that follow one another and with rows of a draft tree (TREE), which differ
// in the keys that a row sees alone.
//
// For a query row i (a token and one of the G query heads of a key head) at
// position p and the keys j it sees (j < len; j <= p if causal; j > p - window)
//   o_i = sum_j w_ij v_j / sum_j w_ij,   w_ij = exp(scale <q_i, k_j>)
// with k_j = ks c_j, v_j = vs d_j: codes c, d of at most 8 significant bits, so
// exact in fp16, and one scale per block of 64 tokens.
//   Scores: q_i is scaled by a power of two so that its largest element is in
//   [2^14, 2^15) and taken in fp16, exactly for elements down to 2^-28 of the
//   largest (bf16 carries 8 bits, fp16 11); products of codes add up in fp32, and
//   score = (scale log2e 2^-x ks) * sum, one factor per row and block.
//   Softmax: running maximum m and sum l per row in fp32, weights 2^(score - m).
//   m is raised, and the sums rescaled, only when a block's maximum passes it by
//   more than kLazy, so weights reach 2^kLazy at most and most blocks skip the
//   rescaling.
//   Values: the block's vs goes into the exponent as r = vs / vref (the
//   accumulators are in units of vref), so it costs nothing per weight:
//   p = 2^(score - m + log2 r + kUp) in fp16 times the codes, added in fp32; l adds
//   (sum of the block's p in fp32) / r.  p rounds to 11 bits (at most 2^-11 of itself;
//   against bf16 weights, 8 bits, an eighth of the error for the same instructions),
//   and kUp keeps weights down to 2^-21 out of fp16's subnormals; smaller ones are off
//   by at most 2^-32, over r.
//   vref is of a row, and of blocks that it sees some token of: raised to a larger
//   vs, lowered to one below 2^-8 vref (value_unit), so r is in [2^-8, 1] however far
//   apart scales lie, and however small the codes that came with the large ones.
//   o is therefore within about 2^-11 max|v| of the exact result before its own
//   rounding to bf16.
#pragma once

#include "kv_cache.hpp"

namespace readme {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));

constexpr float kLazy = 8.0f;  // log2 of the largest weight
constexpr float kUp = 7.0f;    // 2^(kLazy + kUp) = 32768 < 65504, fp16's largest

// Four codes to two fp16 pairs, exact.  int8 bytes are code + 128: 0x64xx is
// 1024 + xx in fp16, less 1152.
template <int KT>
__device__ __forceinline__ void cvt4(uint32_t w, uint32_t& a, uint32_t& b) {
    if constexpr (KT == README_KV_I8) {
        const f16x2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
        const f16x2 lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(w, 0x64646464u, 0x00050004u));
        const f16x2 hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(w, 0x64646464u, 0x00070006u));
        a = __builtin_bit_cast(uint32_t, lo - off);
        b = __builtin_bit_cast(uint32_t, hi - off);
    } else {
        a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, false));
        b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, true));
    }
}
template <int KT>
__device__ __forceinline__ f16x8 cvt8(uint32_t w0, uint32_t w1) {
    u32x4v r;
    uint32_t a, b, c, d;
    cvt4<KT>(w0, a, b);
    cvt4<KT>(w1, c, d);
    r[0] = a;
    r[1] = b;
    r[2] = c;
    r[3] = d;
    return __builtin_bit_cast(f16x8, r);
}

// Bytes of a 16-token piece at or past `n` (tokens that are not in the cache)
// to zero: a byte never written may be an e4m3 NaN, which a weight of zero
// would not silence.
__device__ __forceinline__ uint4 keep_tokens(uint4 w, int n) {
    uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int k = n - 4 * i;
        if (k <= 0) v[i] = 0u;
        else if (k < 4) v[i] &= 0xffffffffu >> (8 * (4 - k));
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// Two weights to fp16, nearest even.
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    const f32x2v p = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(p, f16x2));
}

// Four fp32 to bf16, nearest even (the hardware conversion), 8 bytes.
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint2 pack_bf16(float a, float b, float c, float d) {
    const f32x2v lo = {a, b}, hi = {c, d};
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2v)),
                      __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2v)));
}

// A block's value scale against the row's unit, log_vref = log2 vref: log2 r and
// 1 / r.  At 2^-40 and below every p rounds to zero in fp16: a scale of zero, or one
// that value_unit left that far under the sums.
__device__ __forceinline__ void value_ratio(float vs, float log_vref, float& log_r, float& inv_r) {
    log_r = fmaxf(__builtin_amdgcn_logf(vs) - log_vref, -40.0f);
    inv_r = __builtin_amdgcn_exp2f(-log_r);
}

// The lane's row sees any token of the block at j0.
__device__ __forceinline__ bool sees_block(int lo, int hi, int j0) {
    return max(lo, j0) < min(hi, j0 + kKvBlock);
}

// The unit of a row's sums, for a block of value scale vs.  Lowering multiplies the
// sums, which may hold what a larger scale left: they stop at 2^100 units, and what
// the block adds to sums that large, at most 2^53, is under fp32's rounding of them.
// A unit raised by more than 2^100 may lose them.  A NaN moves nothing.  `row_max`:
// the largest over the lanes that share the row.  Against one unit for the wave, 64
// requests of 2048 tokens and 4 prompts of 2048: value scales within 2^4 of each other
// 44.2 us for 44.1 and 166 for 166; spread over 2^16 44.4 for 44.0 and 173 for 167.
constexpr float kUnitLow = 0x1p-8f;
template <class A, int N, class F>
__device__ __forceinline__ void value_unit(float vs, bool sees, float& vref, float& log_vref, A (&acc)[N],
                                           F&& row_max) {
    const bool up = sees && vs > vref, down = sees && vs > 0.0f && vs < vref * kUnitLow;
    if (!__any(up || down)) return;
    const float ratio = vref * __builtin_amdgcn_rcpf(vs);
    float f = 1.0f, u = vref;
    if (up) {
        f = fminf(ratio, 1.0f);  // at first 0 / vs
        u = vs;
    }
    if (__any(down)) {
        float big = 0.0f;
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int k = 0; k < (int)(sizeof(A) / sizeof(float)); ++k) big = fmaxf(big, fabsf(acc[d][k]));
        big = row_max(big);
        if (down) {
            const float most = fminf(0x1p100f * __builtin_amdgcn_rcpf(big), 0x1p126f);
            f = big == 0.0f ? 1.0f : fminf(ratio, most);
            u = big == 0.0f || ratio <= most ? vs : vref * __builtin_amdgcn_rcpf(most);
        }
    }
    if (up || down) {  // elsewhere vref may be 0 still, with the logarithm 0
        vref = u;
        log_vref = __builtin_amdgcn_logf(u);
    }
#pragma unroll
    for (int d = 0; d < N; ++d) acc[d] *= f;
}

// The scores' factor and offset of a row: 2^(factor * sum + offset) is a weight.
// Both are finite and the factor positive, so that a masked sum of -infinity
// gives 0 also in a row that has seen nothing (m = -infinity).
__device__ __forceinline__ float score_factor(float cq, float ks) { return fmaxf(cq * ks, 1.2e-38f); }
__device__ __forceinline__ float score_offset(float log_r, float m) {
    return log_r + kUp - (m == -INFINITY ? 0.0f : m);
}

// A block whose key or value scale is not finite: every row that sees any of its
// tokens becomes NaN through its sum (the factor and offset above stay finite, so
// other rows' weights for it are 0).
__device__ __forceinline__ bool bad_scales(float ks, float vs) { return !(ks < INFINITY && vs < INFINITY); }

// Token k of a lane's 16 is seen if a0 <= k < a1.
template <class V>
__device__ __forceinline__ void mask_scores(V& v, int a0, int a1) {
#pragma unroll
    for (int k = 0; k < 16; ++k)
        v[k] = (unsigned)(k - a0) < (unsigned)(a1 - a0) ? v[k] : -INFINITY;
}

// Token k of a lane's 16 is seen if bit k is set.
template <class V>
__device__ __forceinline__ void mask_bits(V& v, uint32_t bits) {
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = (bits >> k) & 1u ? v[k] : -INFINITY;
}

// Query rows as fp16 matrix operands.  Each lane holds elements of one row in
// x; `big` is the largest magnitude in the row.  Returns 2^x and its inverse;
// below 2^-100 (a row of zeros among them) the power stays, so that the inverse
// is far from fp32's subnormals.
__device__ __forceinline__ void row_power(float big, float& up, float& down) {
    int e = 0;
    (void)frexpf(big, &e);
    e = big > 0.0f ? e : 0;
    e = e < -100 ? -100 : e;
    up = ldexpf(1.0f, 15 - e);
    down = ldexpf(1.0f, e - 15);
}

// What a request asks of the kernels.
struct KvRequest {
    int64_t row0;     // its first row in the call
    int n;            // its rows
    int len;          // its tokens in the cache
    int block0;       // first and one past the last block any of its rows sees
    int block1;
};

// Request with rows offsets off0 .. off1 and `len` tokens.
__device__ __forceinline__ KvRequest kv_request_of(const KvAttnArgs& a, int64_t off0, int64_t off1,
                                                   int64_t len) {
    KvRequest q;
    int64_t lo, hi;
    kv_clamp_rows(off0, off1, a.c.T, lo, hi);
    q.row0 = lo;
    q.n = (int)(hi - lo);
    const int64_t cap = a.c.max_blocks * kKvBlock;
    const int64_t first = len - q.n;
    int64_t b1 = len < cap ? len : cap;
    b1 = b1 < 0 ? 0 : (b1 + kKvBlock - 1) / kKvBlock;
    int64_t b0 = 0;
    if (a.window > 0 && first - a.window + 1 > 0) b0 = (first - a.window + 1) / kKvBlock;
    q.len = (int)len;
    q.block1 = (int)b1;
    q.block0 = (int)(b0 < b1 ? b0 : b1);
    return q;
}
__device__ __forceinline__ KvRequest kv_request(const KvAttnArgs& a, int64_t r) {
    return kv_request_of(a, a.c.offsets[r], a.c.offsets[r + 1], a.c.lens[r]);
}

// Keys [lo, hi) that a row at position p sees.
__device__ __forceinline__ void row_keys(const KvAttnArgs& a, int len, int64_t p, int& lo, int& hi) {
    int64_t h = a.causal && p + 1 < len ? p + 1 : len;
    int64_t l = a.window > 0 ? p - a.window + 1 : 0;
    h = h < 0 ? 0 : h;
    l = l < 0 ? 0 : (l > h ? h : l);
    lo = (int)l;
    hi = (int)h;
}

// Rows of a draft tree: row t of the request sees the tokens [lo, first) and of the
// request's own rows, at first .. len - 1, those of its bits.  Blocks that all rows
// see whole, between their largest lo and first, ask for no bits.
struct TreeRow {
    int tok;  // -1: there is no row, and what it sees means nothing
    int lo;

    // The given position, where it matters: on its way before set() asks for it.
    __device__ __forceinline__ static int position(const KvAttnArgs& a, const KvRequest& q, int t) {
        return t >= 0 && a.window > 0 && a.pos ? a.pos[q.row0 + t] : 0;
    }
    __device__ __forceinline__ void set(const KvAttnArgs& a, const KvRequest& q, int t, int given) {
        const int64_t first = (int64_t)q.len - q.n;
        tok = t;
        int64_t l = 0;
        if (t >= 0 && a.window > 0) {
            const int64_t p = a.pos ? (int64_t)given : first + t;
            l = (p < first ? first : p) - a.window + 1;
        }
        l = l < first ? l : first;
        lo = (int)(l < 0 ? 0 : l);  // a wide window leaves l far below 32 bits
    }
    // Bit s: the row sees token j0 + s.
    __device__ __forceinline__ uint64_t seen(const KvAttnArgs& a, const KvRequest& q, int j0) const {
        const int f = q.len - q.n - j0;  // the first own row in the block
        uint64_t m = ones_below(f) & ~ones_below(lo - j0);
        if (f < kKvBlock) {
            const uint64_t* bits = a.tree + (q.row0 + (tok < 0 ? 0 : tok)) * a.words;
            uint64_t own;
            if (f > 0) {
                own = bits[0] << f;
            } else {
                const int w = -f >> 6, sh = -f & 63;
                own = w < a.words ? bits[w] >> sh : 0;
                if (sh && w + 1 < a.words) own |= bits[w + 1] << (64 - sh);
            }
            m |= own & ones_below(q.len - j0);
        }
        return m;
    }
    __device__ __forceinline__ static uint64_t ones_below(int n) {
        return n <= 0 ? 0ull : (n >= 64 ? ~0ull : (1ull << n) - 1);
    }
};

// --- dealing the work out -------------------------------------------------------
//
// A pair is (request, tile of query rows, key head); its blocks are those that any
// row of the request sees.  Either a workgroup takes a whole pair, or all pairs, one
// after the other (head fastest), are dealt to the workgroups in contiguous shares
// of equally many blocks, so that one long request among short ones, or few
// requests, fill the chip alike.  Equal in blocks, not in work, where a request has
// many causal rows: blocks past a tile's last row are counted and fetched like the
// others and only their products left out.  Whole pairs of 128 rows stop at the
// tile's own last block; those of 16 rows take all of the request's, products too.
// One causal prompt of 4096 at four heads of 128 takes 81 us (whole pairs of 16
// rows, 13 of needed products), one of 8192 143 (shares of tiles, 51 needed), four of
// 2048 60 (shares, 13 needed).  A pair counts kPairCost units (its start and end) and one
// for each block.  A share may begin and end inside a pair: those ends are
// partial results in the workspace, at most two per workgroup, which a second
// launch joins (k_attention_join); a pair whose blocks are all in one share is
// written at once.
constexpr int kPairCost = 6;

struct KvPlan {
    int64_t weight;  // units of all the request's pairs
    int tiles;
    int blocks;      // of each pair; a pair of none has no units
};

constexpr int kRowsTile = 16;     // query rows of a pair, in the two kernels
constexpr int kTilesTile = 128;
constexpr int kTreeTile = 32;     // and in that of draft trees
constexpr int kRowsShares = 512;  // workgroups that shares are dealt to: two a CU
constexpr int kTilesShares = 512;
constexpr int kTreeShares = 512;

// The order of a request's pairs, and which share a workgroup has.  The draft trees'
// tiles are many to a head and read the same codes: they follow one another, and
// neighbouring shares go to one of the eight dies, whose L2 then holds the codes.
template <int ROWS>
__host__ __device__ constexpr bool kv_tiles_first() {
    return ROWS == kTreeTile;
}
template <int ROWS>
__device__ __forceinline__ int64_t kv_pair_index(int64_t tile, int64_t h, int64_t tiles, int64_t Hk) {
    return kv_tiles_first<ROWS>() ? h * tiles + tile : tile * Hk + h;
}
template <int ROWS>
__device__ __forceinline__ int64_t kv_share_of(int64_t block, int64_t grid) {  // grid a multiple of 8
    return kv_tiles_first<ROWS>() ? (block & 7) * (grid >> 3) + (block >> 3) : block;
}

template <int ROWS>
__device__ __forceinline__ KvPlan kv_plan(const KvAttnArgs& a, const KvRequest& q) {
    KvPlan p;
    p.tiles = (int)(((int64_t)q.n * a.G + ROWS - 1) / ROWS);
    p.blocks = q.block1 - q.block0;
    p.weight = p.blocks > 0 ? (int64_t)p.tiles * a.c.Hk * (p.blocks + kPairCost) : 0;
    return p;
}

// Workspace: int64 [0] units per share, [1 + r] first unit of request r's pairs;
// then the parts, two per workgroup: sums [ROWS][D], then m, l and vref [ROWS]
// (fp32).  The sums stay in units of vref until they are divided by l: they hold
// weights of up to 2^(kLazy + kUp) over all tokens, and times vref would pass fp32's
// largest where the row itself does not.
__host__ __device__ inline int64_t kv_plan_bytes(int64_t R) { return ((R + 1) * 8 + 255) / 256 * 256; }
template <int D, int ROWS>
constexpr int kv_part_floats = ROWS * (D + 3);

// Factor from units of `vref` to units of `most`, the largest of several (0 where
// no block was seen).
__device__ __forceinline__ float unit_ratio(float vref, float most) {
    return most > 0.0f ? vref * __builtin_amdgcn_rcpf(most) : 0.0f;
}

__device__ __forceinline__ int64_t wave_scan64(int64_t v, int lane) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int64_t u = __shfl_up(v, off, 64);
        if (lane >= off) v += u;
    }
    return v;
}

// A value that is the same in all lanes, to scalar registers.
__device__ __forceinline__ int64_t wave_uniform(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)v >> 32));
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

// A workgroup's way through its share, piece by piece.
template <int ROWS, int WAVES>
struct KvWalk {
    int64_t w, w1;     // units left
    int64_t base;      // first unit of request r
    int64_t r, tile;
    int h, b0, nb;     // blocks [b0, b0 + nb) of the pair's
    KvRequest q;
    KvPlan p;
    int64_t me;        // the share's number

    // False if there is no share.  A share is at least `min_share` blocks, or a
    // whole pair where the longest is shorter: cutting finer costs more in parts
    // than it saves.  Workgroup 0 writes the plan down for the join.  `lds`
    // holds 2 WAVES + 2 int64.
    __device__ __forceinline__ bool start(const KvAttnArgs& a, int min_share, int64_t* plan,
                                          int64_t* lds) {
        const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
        const int64_t R = a.c.R, grid = gridDim.x;
        me = kv_share_of<ROWS>(blockIdx.x, gridDim.x);
        int most = 0;  // blocks of the longest pair
        auto weight = [&](int64_t at) {
            if (at >= R) return (int64_t)0;
            const KvPlan k = kv_plan<ROWS>(a, kv_request(a, at));
            if (k.weight > 0) most = max(most, k.blocks);
            return k.weight;
        };
        auto set = [&](int64_t total) {
            int64_t share = (total + grid - 1) / grid;
            const int64_t least = kPairCost + (most < min_share ? most : min_share);
            share = share < least ? least : share;
            share = wave_uniform(share);
            total = wave_uniform(total);
            w = me * share;
            w1 = w + share < total ? w + share : total;
            if (me == 0 && tid == 0) plan[0] = share;
            return w < total;
        };
        auto wave_most = [&]() {
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) most = max(most, __shfl_xor(most, off, 64));
        };
        if (R <= 64) {  // one request a lane, every wave for itself
            const int64_t v = weight(lane), incl = wave_scan64(v, lane), first = incl - v;
            wave_most();
            const bool any = set(__shfl(incl, 63, 64));
            if (me == 0 && wv == 0 && lane < R) plan[1 + lane] = first;
            if (!any) return false;
            const int l = __ffsll((unsigned long long)__ballot(w >= first && w < incl)) - 1;
            r = l;
            base = wave_uniform(__shfl(first, l, 64));
        } else {
            int64_t mine = 0;
            for (int64_t i = tid; i < R; i += WAVES * 64) mine += weight(i);
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) mine += __shfl_xor(mine, off, 64);
            wave_most();
            if (lane == 0) {
                lds[wv] = mine;
                lds[WAVES + 2 + wv] = most;
            }
            __syncthreads();
            int64_t total = 0;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) {
                total += lds[k];
                most = max(most, (int)lds[WAVES + 2 + k]);
            }
            const bool any = set(total);
            if (!any && me != 0) return false;
            int64_t run = 0;
            for (int64_t r0 = 0; r0 < R; r0 += WAVES * 64) {
                const int64_t i = r0 + tid;
                const int64_t v = weight(i), incl = wave_scan64(v, lane);
                __syncthreads();
                if (lane == 63) lds[wv] = incl;
                __syncthreads();
                int64_t first = run + incl - v;
#pragma unroll
                for (int k = 0; k < WAVES; ++k) {
                    if (k < wv) first += lds[k];
                    run += lds[k];
                }
                if (w >= first && w < first + v) {
                    lds[WAVES] = i;
                    lds[WAVES + 1] = first;
                }
                if (me == 0 && i < R) plan[1 + i] = first;
                if (me != 0 && run > w) break;
            }
            if (!any) return false;
            __syncthreads();
            r = wave_uniform(lds[WAVES]);
            base = wave_uniform(lds[WAVES + 1]);
        }
        q = kv_request(a, r);
        p = kv_plan<ROWS>(a, q);
        return true;
    }

    // The next piece with blocks; false at the share's end.
    __device__ __forceinline__ bool next(const KvAttnArgs& a) {
        while (w < w1) {
            while (w >= base + p.weight) {  // ends: w is below the sum of all weights
                base += p.weight;
                q = kv_request(a, ++r);
                p = kv_plan<ROWS>(a, q);
            }
            const int64_t units = p.blocks + kPairCost;
            const int64_t pair = (w - base) / units;
            const int u0 = (int)((w - base) - pair * units);
            const int u1 = w1 - w < units - u0 ? u0 + (int)(w1 - w) : (int)units;
            w += u1 - u0;
            b0 = u0 > kPairCost ? u0 - kPairCost : 0;
            nb = (u1 > kPairCost ? u1 - kPairCost : 0) - b0;
            if constexpr (kv_tiles_first<ROWS>()) {
                h = (int)(pair / p.tiles);
                tile = pair - (int64_t)h * p.tiles;
            } else {
                tile = pair / a.c.Hk;
                h = (int)(pair - tile * a.c.Hk);
            }
            if (nb > 0) return true;
        }
        return false;
    }

    __device__ __forceinline__ bool whole() const { return nb == p.blocks; }
    // The pair begins in this share, or before it.
    __device__ __forceinline__ int64_t part() const { return me * 2 + (b0 == 0 ? 1 : 0); }
};

// Tile j of request r is slot floor(offsets[r] G / ROWS) + r + j, which needs no
// sum over the requests (and leaves some slots empty): the request of a slot,
// and the tile.  The last step of the search has one request a lane and loads all
// of it, one dependent load less.
template <int ROWS>
__device__ __forceinline__ KvRequest kv_slot_request(const KvAttnArgs& a, int64_t slot, int64_t& r,
                                                     int64_t& tile) {
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, n = a.c.R;
    while (n > 64) {
        const int64_t step = (n + 63) / 64, i = lane * step;
        const bool le = i < n && (int64_t)a.c.offsets[lo + i] * a.G / ROWS + lo + i <= slot;
        const int below = __popcll(__ballot(le));
        const int64_t skip = below > 0 ? (int64_t)(below - 1) * step : 0;
        lo += skip;
        n = n - skip < step ? n - skip : step;
    }
    int off0 = 0, off1 = 0, len = 0;
    if (lane < n) {
        off0 = a.c.offsets[lo + lane];
        off1 = a.c.offsets[lo + lane + 1];
        len = a.c.lens[lo + lane];
    }
    const bool le = lane < n && (int64_t)off0 * a.G / ROWS + lo + lane <= slot;
    const int below = __popcll(__ballot(le)), l = below > 0 ? below - 1 : 0;
    off0 = __builtin_amdgcn_readlane(off0, l);
    off1 = __builtin_amdgcn_readlane(off1, l);
    len = __builtin_amdgcn_readlane(len, l);
    r = lo + l;
    tile = slot - ((int64_t)off0 * a.G / ROWS + r);
    return kv_request_of(a, off0, off1, len);
}
__host__ __device__ inline int64_t kv_slots(int64_t T, int64_t R, int64_t G, int rows) { return T * G / rows + R; }

// One lane's block number and scales: block j of request r (-1: absent).
struct KvBlockRef {
    int blk;
    float ks, vs;
};
// The block's scales as they are stored, and as the kernels take them.
__device__ __forceinline__ float2 kv_block_scales(const KvAttnArgs& a, int blk, int h) {
    if (blk < 0) return make_float2(0.0f, 0.0f);
    return *reinterpret_cast<const float2*>(a.c.scales + ((int64_t)blk * a.c.Hk + h) * 2);
}
__device__ __forceinline__ void kv_set_scales(KvBlockRef& b, float2 sc) {
    // An infinite scale counts as NaN: its logarithm and products of a score
    // of zero are not numbers.
    const bool bad = bad_scales(sc.x, sc.y);
    b.ks = bad ? __builtin_nanf("") : sc.x;
    // No scale that the write gives is subnormal; one counts as zero, since its
    // reciprocal is infinite.
    b.vs = bad ? __builtin_nanf("") : sc.y < 0x1p-126f ? 0.0f : sc.y;
}
__device__ __forceinline__ KvBlockRef kv_block_ref(const KvAttnArgs& a, int64_t r, int64_t j, int h) {
    KvBlockRef b;
    b.blk = (int)kv_block_of(a.c.table, a.c.max_blocks, a.c.n_blocks, r, j);
    kv_set_scales(b, kv_block_scales(a, b.blk, h));
    return b;
}
__device__ __forceinline__ KvBlockRef kv_lane_ref(const KvBlockRef& b, int lane) {
    KvBlockRef o;
    o.blk = __builtin_amdgcn_readlane(b.blk, lane);
    o.ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(b.ks), lane));
    o.vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(b.vs), lane));
    return o;
}

// `waves` of a workgroup that takes a whole pair (1, 2, 4, 8), or 0 for shares.
hipError_t launch_attention_rows(readme_kv_type kt, const KvAttnArgs& a, int waves, hipStream_t s);
hipError_t launch_attention_tiles(readme_kv_type kt, const KvAttnArgs& a, bool shares, hipStream_t s);
// The same with a.tree.
hipError_t launch_attention_tree(readme_kv_type kt, const KvAttnArgs& a, int waves, hipStream_t s);
hipError_t launch_attention_tree_rows(readme_kv_type kt, const KvAttnArgs& a, int waves, hipStream_t s);
hipError_t launch_attention_tree_tiles(readme_kv_type kt, const KvAttnArgs& a, bool shares, hipStream_t s);

}  // namespace readme
