// Writing rows into the 8-bit cache: how a call's blocks are found, how codes are
// made, and one block's write.  Shared by kv_cache.hip (rows as they are) and
// kv_append.hip (keys turned on the way); kv_cache.hip has the mathematics.
#pragma once

#include <math.h>

#include "kv_cache.hpp"
#include "rotary.hpp"

namespace readme {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// 16 consecutive values of a row, as they are stored.
template <int DT>
struct Row16 {
    uint4 v[DT == README_BF16 ? 2 : 4];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (auto& x : v) x = make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ __forceinline__ void load(const void* base, int64_t at) {
        const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(base) +
                                                        at * (DT == README_BF16 ? 2 : 4));
#pragma unroll
        for (auto& x : v) x = *p++;
    }
    __device__ __forceinline__ float at(int k) const {
        const int d = DT == README_BF16 ? k >> 1 : k;
        const uint4 q = v[d >> 2];
        const uint32_t w = (d & 3) == 0 ? q.x : (d & 3) == 1 ? q.y : (d & 3) == 2 ? q.z : q.w;
        if constexpr (DT == README_F32) return __uint_as_float(w);
        return k & 1 ? bf16_hi(w) : bf16_lo(w);
    }
    // Bits of the largest magnitude, a NaN above every number.
    __device__ __forceinline__ uint32_t most() const {
        if constexpr (DT == README_F32) {
            uint32_t m = 0;
#pragma unroll
            for (auto& q : v)
                m = max(m, max(max(q.x & 0x7fffffffu, q.y & 0x7fffffffu),
                               max(q.z & 0x7fffffffu, q.w & 0x7fffffffu)));
            return m;
        } else {
            u16x2 m = {0, 0};
#pragma unroll
            for (auto& q : v)
#pragma unroll
                for (const uint32_t w : {q.x, q.y, q.z, q.w})
                    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w & 0x7fff7fffu));
            return (uint32_t)(m[0] > m[1] ? m[0] : m[1]) << 16;
        }
    }
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <int DT>
__device__ __forceinline__ void store16(void* base, int64_t at, const float (&x)[16]) {
    if constexpr (DT == README_BF16) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {  // the hardware conversion, nearest even
            const f32x2 p = {x[2 * i], x[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
        }
        uint4* p = reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(base) + at);
        p[0] = make_uint4(w[0], w[1], w[2], w[3]);
        p[1] = make_uint4(w[4], w[5], w[6], w[7]);
    } else {
        float4* p = reinterpret_cast<float4*>(reinterpret_cast<float*>(base) + at);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            p[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    }
}

__device__ __forceinline__ uint32_t e4m3_byte(float x) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, 0.0f, 0, false) & 0xffu;
}

// x / s (inv = 1 / s in fp32) rounded to odd: one Newton step makes q faithful
// (less than one unit off), the sign of x - q s tells on which side x / s lies,
// and taking the neighbour with an odd last bit keeps a second rounding, to e4m3,
// from seeing a tie where there is none.
__device__ __forceinline__ float quotient_odd(float x, float s, float inv) {
    float q = x * inv;
    q = fmaf(fmaf(-q, s, x), inv, q);
    const float r = fmaf(-q, s, x);
    uint32_t u = __float_as_uint(q);
    if (r != 0.0f && !(u & 1u)) u = ((r > 0.0f) == (q > 0.0f)) ? u + 1u : u - 1u;
    if (q == 0.0f) u = 0u;
    return __uint_as_float(u);
}

// The int8 code nearest to x / s, plus 128, ties to even: n = rint(x inv) is at
// most one off; x - n s is exact in fp32 (a multiple of s's last place and at
// most 1.5 s, or x near s), so comparing it with s / 2 settles n.
__device__ __forceinline__ uint32_t nearest_i8(float x, float s, float inv) {
    float n = rintf(x * inv);
    const float r = fmaf(-n, s, x), h = 0.5f * s;
    const bool odd = ((int)n & 1) != 0;
    if (r > h || (r == h && odd)) n += 1.0f;
    else if (r < -h || (r == -h && odd)) n -= 1.0f;
    n = fminf(fmaxf(n, -127.0f), 127.0f);
    return (uint32_t)((int)n + 128);
}

// Codes of a row's 16 values.  The plain product q = x inv is within 2 units in
// its last place of x / s, so its nearest code is the quotient's unless a tie
// between two codes lies that near.  Such values are settled one by one: bf16
// rows hold many ties of one kind (half of the largest element is 63.5 int8
// codes), so a whole row would rarely go without.  The write of 16155 rows of 8
// heads of 128 takes 27 us this way, 36 with rows settled whole, 33 with every
// value settled.
//   int8: adding 1.5 2^23 rounds q to an integer, ties to even, and leaves code
//   + 128 in the low byte; |q| <= 127, so 2 units are at most 2^-16.
//   e4m3: from 2^-6 on a tie is the middle of the 20 mantissa bits that a code
//   does not have; smaller quotients all go the long way.
template <int KT, int DT>
__device__ __forceinline__ void encode16(const Row16<DT>& x, float s, float inv, uint32_t (&w)[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (KT == README_KV_I8) {
            constexpr float kRound = 12582912.0f + 128.0f;
            uint32_t u[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = x.at(4 * k + e), q = v * inv, f = q + kRound;
                u[e] = __float_as_uint(f);
                if (fabsf(q - (f - kRound)) > 0.5f - 0x1p-15f) u[e] = nearest_i8(v, s, inv);
            }
            w[k] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(u[3], u[2], 0x0c0c0400u),
                                         __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), 0x05040100u);
        } else {
            float c[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = x.at(4 * k + e), q = v * inv;
                c[e] = q;
                if (((__float_as_uint(q) + 0x80003u) & 0xfffffu) <= 6u || fabsf(q) < 0x1p-6f)
                    c[e] = quotient_odd(v, s, inv);
                c[e] = fminf(fmaxf(c[e], -448.0f), 448.0f);
            }
            const int b = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
            w[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], b, true);
        }
    }
}

// Four codes times s.
template <int KT>
__device__ __forceinline__ void decode4(uint32_t w, float s, float* x) {
    if constexpr (KT == README_KV_I8) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (float)((int)((w >> (8 * e)) & 0xffu) - 128) * s;
    } else {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
        const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        x[0] = a[0] * s;
        x[1] = a[1] * s;
        x[2] = b[0] * s;
        x[3] = b[1] * s;
    }
}
// The code nearest to a code's value times f (ties to even).
template <int KT>
__device__ __forceinline__ uint32_t regrid(uint32_t b, float f) {
    if constexpr (KT == README_KV_I8) return (uint32_t)((int)rintf((float)((int)b - 128) * f) + 128);
    return e4m3_byte(__builtin_amdgcn_cvt_f32_fp8((int)b, 0) * f);
}
template <int KT>
__device__ __forceinline__ uint32_t regrid4(uint32_t w, float f) {
    return regrid<KT>(w & 0xffu, f) | (regrid<KT>((w >> 8) & 0xffu, f) << 8) |
           (regrid<KT>((w >> 16) & 0xffu, f) << 16) | (regrid<KT>(w >> 24, f) << 24);
}

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        const uint32_t u = (uint32_t)__shfl_xor((int)v, off, 64);
        v = u > v ? u : v;
    }
    return v;
}

// One (request, block) that a call's rows lie in: rows tok .. tok + n - 1 at
// slots slot .. slot + n - 1 of the request's block j.
struct Touched {
    int64_t r, j, tok;
    int slot, n;
};

__device__ __forceinline__ Touched touched(const KvCacheArgs& c, int64_t r, int64_t lo, int64_t hi,
                                           int64_t tok) {
    const int64_t p = (int64_t)c.lens[r] - (hi - tok);
    Touched b;
    b.r = r;
    b.tok = tok;
    b.j = kv_block_index(p);
    b.slot = kv_slot(p);
    b.n = (int)(hi - tok < kKvBlock - b.slot ? hi - tok : kKvBlock - b.slot);
    return b;
}

// Calls f(Touched) for every block of candidate `cand` (uniform over the
// wave): cand < R the first block of request cand, else the blocks that begin
// at rows 64 (cand - R) .. + 63 and are not their request's first.  With `apart` a
// request's second block is a candidate of its own too, after the R first ones: of
// requests of fewer than 64 rows several begin one within a run of 64 rows and would
// follow one another, while of third and later blocks a run has at most one.
template <class F>
__device__ __forceinline__ void for_touched(const KvCacheArgs& c, int64_t cand, bool apart, F&& f) {
    const int64_t alone = apart ? 2 * c.R : c.R;
    if (cand < alone) {
        const bool second = cand >= c.R;
        const int64_t r = second ? cand - c.R : cand;
        int64_t lo, hi;
        kv_rows(c.offsets, c.T, r, lo, hi);
        int64_t tok = lo;
        if (second) tok += kKvBlock - kv_slot((int64_t)c.lens[r] - (hi - lo));
        if (tok < hi) f(touched(c, r, lo, hi, tok));
        return;
    }
    const int lane = threadIdx.x & 63;
    const int64_t t0 = (cand - alone) * kKvBlock;
    const int64_t t1 = t0 + kKvBlock < c.T ? t0 + kKvBlock : c.T;
    for (int64_t r0 = kv_request_at(c.offsets, c.R, t0); r0 < c.R; r0 += 64) {
        // Lane l looks at request r0 + l: does a block of it begin in the run?
        int64_t lo = c.T, hi = c.T, tok = -1;
        if (r0 + lane < c.R) {
            kv_rows(c.offsets, c.T, r0 + lane, lo, hi);
            const int64_t p = (int64_t)c.lens[r0 + lane] - (hi - lo);
            int64_t b = lo + (apart ? 2 : 1) * kKvBlock - kv_slot(p);
            if (b < t0) b += (t0 - b + kKvBlock - 1) / kKvBlock * kKvBlock;
            if (b < t1 && b < hi) tok = b;
        }
        uint64_t hit = __ballot(tok >= 0);
        while (hit) {
            const int l = __ffsll((unsigned long long)hit) - 1;
            hit &= hit - 1;
            const int64_t rl = __shfl(lo, l, 64), rh = __shfl(hi, l, 64), tk = __shfl(tok, l, 64);
            f(touched(c, r0 + l, rl, rh, tk));
        }
        if (__ballot(lo >= t1) != 0) break;  // offsets do not decrease
    }
}

constexpr int kKvThreads = 256;
// Passes over a block's 64 rows.
template <int D>
constexpr int kKvPasses = kKvBlock * (D / 16) / kKvThreads;
// LDS holds a block's V codes as 64 token rows, one dword apart so that a
// column's dwords spread over the banks.
constexpr int kv_lds_row(int D) { return D / 4 + 1; }

// Four dwords of four bytes each, transposed: byte j of out[i] is byte i of
// in[j].
__device__ __forceinline__ void transpose4(const uint32_t (&in)[4], uint32_t (&out)[4]) {
    const uint32_t a = __builtin_amdgcn_perm(in[1], in[0], 0x05010400u);  // 0.0 1.0 0.1 1.1
    const uint32_t b = __builtin_amdgcn_perm(in[1], in[0], 0x07030602u);  // 0.2 1.2 0.3 1.3
    const uint32_t c = __builtin_amdgcn_perm(in[3], in[2], 0x05010400u);
    const uint32_t d = __builtin_amdgcn_perm(in[3], in[2], 0x07030602u);
    out[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
    out[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    out[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    out[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// A thread's part of a V block in memory: eight tokens t0 .. t0 + 7 of four
// dims d0 .. d0 + 3, as two dwords a dim.  Item i of 2 D; four neighbours make
// a dim's 32 bytes.
struct VPiece {
    int t0, d0;
};
__device__ __forceinline__ VPiece v_piece(int D, int i) {
    VPiece p;
    p.t0 = (i / D) * 32 + (i & 3) * 8;
    p.d0 = (i % D >> 2) * 4;
    return p;
}

// The rows of a call as write_block takes them: sixteen dims d0 .. d0 + 15 of a
// row as they are.
template <int DT>
struct PlainRows {
    static constexpr int kType = DT;       // of the values
    static constexpr bool kOneRun = true;  // the dims follow one another
    typedef Row16<DT> Raw;
    const void* base;
    int64_t ld;
    __device__ __forceinline__ void zero(Raw& x) const { x.zero(); }
    __device__ __forceinline__ void load(Raw& x, const Touched& b, int row, int col, int ch) const {
        x.load(base, (b.tok + row) * ld + col + ch * 16);
    }
    __device__ __forceinline__ Row16<DT> value(const Raw& x, const Touched&, int, int) const { return x; }
};

// One block of K or V, by the whole workgroup: a thread holds 16 values of a
// row per pass, the rows stay in registers between the maximum and the codes.
template <int KT, int D, bool V, class Rows>
__device__ __forceinline__ void write_block(const KvCacheArgs& c, const Touched& b, int h,
                                            const Rows& src, uint32_t* lds, uint32_t* most) {
    constexpr int DT = Rows::kType;
    const int64_t blk = kv_block_of(c.table, c.max_blocks, c.n_blocks, b.r, b.j);
    if (blk < 0) return;
    const int tid = threadIdx.x, lane = tid & 63;
    constexpr int LPR = D / 16;           // threads per row
    constexpr int RPP = kKvThreads / LPR;   // rows per pass
    constexpr int NP = kKvPasses<D>;
    const int ch = tid % LPR, rw = tid / LPR;
    const int64_t unit = (blk * c.Hk + h) * 2 + (V ? 1 : 0);
    uint8_t* dst = c.codes + unit * kv_half_bytes(D);
    const float old = b.slot > 0 ? c.scales[unit] : 1.0f;

    typename Rows::Raw raw[NP];
    Row16<DT> x[NP];
    uint32_t am = 0;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        src.zero(raw[p]);
        if (p * RPP + rw < b.n) src.load(raw[p], b, p * RPP + rw, h * D, ch);
    }
#pragma unroll
    for (int p = 0; p < NP; ++p) x[p] = src.value(raw[p], b, p * RPP + rw, ch);
#pragma unroll
    for (int p = 0; p < NP; ++p) am = max(am, x[p].most());
    am = wave_max_u32(am);
    __syncthreads();  // an earlier block's reads of `most` and `lds` are over
    if (lane == 0) most[tid >> 6] = am;
    __syncthreads();
    am = max(max(most[0], most[1]), max(most[2], most[3]));

    const float need = __uint_as_float(am) / kv_qmax<KT>();
    float s = fmaxf(need, kKvScaleFloor), shrink = 1.0f;
    bool bad = am >= 0x7f800000u;
    if (b.slot > 0) {
        int e_need, e_old;
        (void)frexpf(need, &e_need);
        const float m = frexpf(old, &e_old);
        int k = need > 0.0f ? e_need - e_old : 0;
        if (k < 0) k = 0;
        if (ldexpf(old, k) < need) ++k;
        s = ldexpf(old, k);
        shrink = ldexpf(1.0f, -k);
        bad = bad || !(m > 0.0f && m < 1.0f);   // NaN (or a scale never written)
    }
    if (bad) {
        s = __uint_as_float(0x7fc00000u);
        shrink = 1.0f;
    }
    const bool grown = shrink != 1.0f;
    if (tid == 0) c.scales[unit] = s;
    const float inv = 1.0f / s;

    if constexpr (!V) {
        if (grown) {
            for (int i = tid; i < b.slot * LPR; i += kKvThreads) {
                uint4* p = reinterpret_cast<uint4*>(dst + kv_k_byte(D, i / LPR, (i % LPR) * 16));
                uint4 w = *p;
                w.x = regrid4<KT>(w.x, shrink);
                w.y = regrid4<KT>(w.y, shrink);
                w.z = regrid4<KT>(w.z, shrink);
                w.w = regrid4<KT>(w.w, shrink);
                *p = w;
            }
        }
    }
    // Few rows of V go byte by byte, more (and a block whose earlier codes
    // change) through LDS.
    const bool staged = V && (grown || b.n > 4);
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int i = p * RPP + rw;
        if (i >= b.n) break;
        uint32_t w[4];
        encode16<KT, DT>(x[p], s, inv, w);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (bad) w[k] = KT == README_KV_I8 ? 0x80808080u : 0u;
        if constexpr (!V && Rows::kOneRun) {
            *reinterpret_cast<uint4*>(dst + kv_k_byte(D, b.slot + i, ch * 16)) =
                make_uint4(w[0], w[1], w[2], w[3]);
        } else if constexpr (!V) {
            const Chunk k = src.chunk(ch);
            *reinterpret_cast<uint2*>(dst + kv_k_byte(D, b.slot + i, k.a)) = make_uint2(w[0], w[1]);
            *reinterpret_cast<uint2*>(dst + kv_k_byte(D, b.slot + i, k.b)) = make_uint2(w[2], w[3]);
        } else if (staged) {
#pragma unroll
            for (int k = 0; k < 4; ++k) lds[(b.slot + i) * kv_lds_row(D) + ch * 4 + k] = w[k];
        } else {
#pragma unroll
            for (int k = 0; k < 16; ++k)
                dst[kv_v_byte(D, b.slot + i, ch * 16 + k)] = (uint8_t)(w[k >> 2] >> (8 * (k & 3)));
        }
    }
    if constexpr (V) {
        if (!staged) return;
        __syncthreads();
        const int end = b.slot + b.n;
        for (int i = tid; i < 2 * D; i += kKvThreads) {
            const VPiece v = v_piece(D, i);
            if (v.t0 >= end || (v.t0 + 8 <= b.slot && !grown)) continue;
            uint32_t in[2][4], out[2][4];
#pragma unroll
            for (int e = 0; e < 8; ++e) in[e >> 2][e & 3] = lds[(v.t0 + e) * kv_lds_row(D) + v.d0 / 4];
            transpose4(in[0], out[0]);
            transpose4(in[1], out[1]);
            uint8_t* at = dst + kv_v_byte(D, v.t0, v.d0);
            if (v.t0 >= b.slot && v.t0 + 8 <= end) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    *reinterpret_cast<uint2*>(at + 32 * k) = make_uint2(out[0][k], out[1][k]);
            } else {
                // Earlier tokens keep their (rescaled) codes, later bytes theirs.
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint2 was = *reinterpret_cast<const uint2*>(at + 32 * k);
                    uint32_t w[2] = {was.x, was.y};
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int t = v.t0 + e, sh = 8 * (e & 3);
                        uint32_t byte = (w[e >> 2] >> sh) & 0xffu;
                        if (t >= b.slot && t < end) byte = (out[e >> 2][k] >> sh) & 0xffu;
                        else if (t < b.slot && grown) byte = regrid<KT>(byte, shrink);
                        w[e >> 2] = (w[e >> 2] & ~(0xffu << sh)) | (byte << sh);
                    }
                    *reinterpret_cast<uint2*>(at + 32 * k) = make_uint2(w[0], w[1]);
                }
            }
        }
    }
}

// K (z = 0) or V of candidate blockIdx.x, head blockIdx.y.
template <int KT, int D, class KRows, class VRows>
__device__ __forceinline__ void write_candidate(const KvCacheArgs& c, bool apart, KRows k, VRows v) {
    __shared__ uint32_t lds[kKvBlock * kv_lds_row(D)];
    __shared__ uint32_t most[4];
    const int h = blockIdx.y;
    if (blockIdx.z)
        for_touched(c, blockIdx.x, apart, [&](const Touched& b) {
            write_block<KT, D, true>(c, b, h, v, lds, most);
        });
    else
        for_touched(c, blockIdx.x, apart, [&](const Touched& b) {
            write_block<KT, D, false>(c, b, h, k, lds, most);
        });
}
inline dim3 kv_grid(const KvCacheArgs& c) {
    return dim3((unsigned)(c.R + ceil_div(c.T, kKvBlock)), (unsigned)c.Hk, 2u);
}

// L<code type, row type, head dims>::go(a...) of a call's types.
template <template <int, int, int> class L, class... A>
inline hipError_t by_type(readme_kv_type kt, readme_dtype dt, int D, A... a) {
    const int at = (kt == README_KV_I8 ? 0 : 2) + (dt == README_F32 ? 0 : 1);
    switch (D * 4 + at) {
        case 64 * 4 + 0: return L<README_KV_I8, README_F32, 64>::go(a...);
        case 64 * 4 + 1: return L<README_KV_I8, README_BF16, 64>::go(a...);
        case 64 * 4 + 2: return L<README_KV_E4M3, README_F32, 64>::go(a...);
        case 64 * 4 + 3: return L<README_KV_E4M3, README_BF16, 64>::go(a...);
        case 128 * 4 + 0: return L<README_KV_I8, README_F32, 128>::go(a...);
        case 128 * 4 + 1: return L<README_KV_I8, README_BF16, 128>::go(a...);
        case 128 * 4 + 2: return L<README_KV_E4M3, README_F32, 128>::go(a...);
        case 128 * 4 + 3: return L<README_KV_E4M3, README_BF16, 128>::go(a...);
        case 256 * 4 + 0: return L<README_KV_I8, README_F32, 256>::go(a...);
        case 256 * 4 + 1: return L<README_KV_I8, README_BF16, 256>::go(a...);
        case 256 * 4 + 2: return L<README_KV_E4M3, README_F32, 256>::go(a...);
        case 256 * 4 + 3: return L<README_KV_E4M3, README_BF16, 256>::go(a...);
    }
    return hipErrorInvalidValue;
}

}  // namespace readme
