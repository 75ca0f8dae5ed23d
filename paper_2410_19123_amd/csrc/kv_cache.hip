// Writing rows into the 8-bit key/value cache and reading them back
// (readme_kv_write, readme_kv_read).
//
// One scale s per (block of 64 tokens, head, K or V); a value is code * s.
//   a block without earlier rows   s = max(amax / QMAX, 2^-100)
//   a block with earlier rows      s = s_old * 2^k, the least k >= 0 with
//                                  amax(new rows) / QMAX <= s
// and the earlier codes become round(code * 2^-k).  Growing by powers of two
// keeps that step exact up to its one rounding, so however often a block
// grows an earlier value moves by less than one step of the final scale
// (1/2 + 1/4 + ...); a scale that followed amax itself would add half a step
// at every growth.  A prompt's blocks are written whole and get the tight
// scale.  New codes are the nearest to the real quotient x / s, ties to even.
// A block that receives an infinity or a NaN gets the scale NaN, so that every
// value read from it is NaN, and keeps it until it is written anew.
//
// Which blocks a call touches is not known on the host.  Every touched block
// is either the first of its request in this call (one candidate per request)
// or begins at one of the call's rows; a request has at most one such row in a
// run of 64, so a workgroup per run of 64 rows finds them.  Both kernels run
// one workgroup per (candidate, head, K or V) and need no plan and no workspace.
// K's rows become 16-byte pieces as they are; V's tokens lie beside each other in
// a block, so its codes pass through LDS, four bytes transposed in registers.
// Measured: reading 105275 rows of 8 heads of 128 from int8 to bf16, 647 MB in
// 137 us, 4.7 TB/s, a large copy's rate (4.9); writing 16155 such rows from bf16
// to e4m3, 99 MB in 27 us, 3.6 TB/s, held by the conversion's instructions; a row
// each of 64 requests 5.5 us to write (3 more where every block grows) and 7 to read
// the blocks back: launch, the search of the request, one dependent load each of
// table, scale and codes.
#include <math.h>

#include "kv_cache.hpp"

namespace readme {

namespace {

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
// at rows 64 (cand - R) .. + 63 and are not their request's first.
template <class F>
__device__ __forceinline__ void for_touched(const KvCacheArgs& c, int64_t cand, F&& f) {
    if (cand < c.R) {
        int64_t lo, hi;
        kv_rows(c.offsets, c.T, cand, lo, hi);
        if (lo < hi) f(touched(c, cand, lo, hi, lo));
        return;
    }
    const int lane = threadIdx.x & 63;
    const int64_t t0 = (cand - c.R) * kKvBlock;
    const int64_t t1 = t0 + kKvBlock < c.T ? t0 + kKvBlock : c.T;
    for (int64_t r0 = kv_request_at(c.offsets, c.R, t0); r0 < c.R; r0 += 64) {
        // Lane l looks at request r0 + l: does a block of it begin in the run?
        int64_t lo = c.T, hi = c.T, tok = -1;
        if (r0 + lane < c.R) {
            kv_rows(c.offsets, c.T, r0 + lane, lo, hi);
            const int64_t p = (int64_t)c.lens[r0 + lane] - (hi - lo);
            int64_t b = lo + kKvBlock - kv_slot(p);
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

constexpr int kThreads = 256;
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

// One block of K or V, by the whole workgroup: a thread holds 16 values of a
// row per pass, the rows stay in registers between the maximum and the codes.
template <int KT, int DT, int D, bool V>
__device__ __forceinline__ void write_block(const KvCacheArgs& c, const Touched& b, int h,
                                            const void* src, int64_t ld, uint32_t* lds,
                                            uint32_t* most) {
    const int64_t blk = kv_block_of(c.table, c.max_blocks, c.n_blocks, b.r, b.j);
    if (blk < 0) return;
    const int tid = threadIdx.x, lane = tid & 63;
    constexpr int LPR = D / 16;           // threads per row
    constexpr int RPP = kThreads / LPR;   // rows per pass
    constexpr int NP = kKvBlock / RPP;
    const int ch = tid % LPR, rw = tid / LPR;
    const int64_t unit = (blk * c.Hk + h) * 2 + (V ? 1 : 0);
    uint8_t* dst = c.codes + unit * kv_half_bytes(D);
    const int64_t col = (int64_t)h * D + ch * 16;
    const float old = b.slot > 0 ? c.scales[unit] : 1.0f;

    Row16<DT> x[NP];
    uint32_t am = 0;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        x[p].zero();
        if (p * RPP + rw < b.n) x[p].load(src, (b.tok + p * RPP + rw) * ld + col);
    }
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
            for (int i = tid; i < b.slot * LPR; i += kThreads) {
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
        if constexpr (!V) {
            *reinterpret_cast<uint4*>(dst + kv_k_byte(D, b.slot + i, ch * 16)) =
                make_uint4(w[0], w[1], w[2], w[3]);
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
        for (int i = tid; i < 2 * D; i += kThreads) {
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

// K (blockIdx.z = 0) or V of (candidate blockIdx.x, head blockIdx.y).
template <int KT, int DT, int D>
__global__ __launch_bounds__(kThreads) void k_kv_write(KvCacheArgs c, const void* __restrict__ k,
                                                       int64_t ld_k, const void* __restrict__ v,
                                                       int64_t ld_v) {
    __shared__ uint32_t lds[kKvBlock * kv_lds_row(D)];
    __shared__ uint32_t most[4];
    const int h = blockIdx.y;
    if (blockIdx.z)
        for_touched(c, blockIdx.x, [&](const Touched& b) {
            write_block<KT, DT, D, true>(c, b, h, v, ld_v, lds, most);
        });
    else
        for_touched(c, blockIdx.x, [&](const Touched& b) {
            write_block<KT, DT, D, false>(c, b, h, k, ld_k, lds, most);
        });
}

template <int KT, int DT, int D, bool V>
__device__ __forceinline__ void read_block(const KvCacheArgs& c, const Touched& b, int h, void* out,
                                           int64_t ld, uint32_t* lds) {
    const int tid = threadIdx.x;
    constexpr int LPR = D / 16, RPP = kThreads / LPR, NP = kKvBlock / RPP;
    const int ch = tid % LPR, rw = tid / LPR;
    const int64_t blk = kv_block_of(c.table, c.max_blocks, c.n_blocks, b.r, b.j);
    const int64_t unit = blk < 0 ? 0 : (blk * c.Hk + h) * 2 + (V ? 1 : 0);
    const uint8_t* src = c.codes + unit * kv_half_bytes(D);
    const float s = blk < 0 ? 0.0f : c.scales[unit];
    const int64_t col = (int64_t)h * D + ch * 16;
    uint32_t w[NP][4];
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int k = 0; k < 4; ++k) w[p][k] = KT == README_KV_I8 ? 0x80808080u : 0u;
    if constexpr (V) {
        if (blk >= 0) {
            constexpr int NI = 2 * D / kThreads > 0 ? 2 * D / kThreads : 1;
            uint32_t in[NI][2][4];
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int i = tid + j * kThreads;
                if (i >= 2 * D) break;
                const VPiece v = v_piece(D, i);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint2 a = *reinterpret_cast<const uint2*>(src + kv_v_byte(D, v.t0, v.d0 + k));
                    in[j][0][k] = a.x;
                    in[j][1][k] = a.y;
                }
            }
            __syncthreads();  // an earlier block's reads are over
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int i = tid + j * kThreads;
                if (i >= 2 * D) break;
                const VPiece v = v_piece(D, i);
                uint32_t o[4];
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    transpose4(in[j][q], o);
#pragma unroll
                    for (int e = 0; e < 4; ++e) lds[(v.t0 + 4 * q + e) * kv_lds_row(D) + v.d0 / 4] = o[e];
                }
            }
            __syncthreads();
#pragma unroll
            for (int p = 0; p < NP; ++p)
                if (p * RPP + rw < b.n)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        w[p][k] = lds[(b.slot + p * RPP + rw) * kv_lds_row(D) + ch * 4 + k];
        }
    } else if (blk >= 0) {
#pragma unroll
        for (int p = 0; p < NP; ++p)
            if (p * RPP + rw < b.n) {
                const uint4 a = *reinterpret_cast<const uint4*>(
                    src + kv_k_byte(D, b.slot + p * RPP + rw, ch * 16));
                w[p][0] = a.x;
                w[p][1] = a.y;
                w[p][2] = a.z;
                w[p][3] = a.w;
            }
    }
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        if (p * RPP + rw >= b.n) break;
        float x[16];
#pragma unroll
        for (int k = 0; k < 4; ++k) decode4<KT>(w[p][k], s, &x[4 * k]);
        store16<DT>(out, (b.tok + p * RPP + rw) * ld + col, x);
    }
}

template <int KT, int DT, int D>
__global__ __launch_bounds__(kThreads) void k_kv_read(KvCacheArgs c, void* __restrict__ k, int64_t ld_k,
                                                      void* __restrict__ v, int64_t ld_v) {
    __shared__ uint32_t lds[kKvBlock * kv_lds_row(D)];
    const int h = blockIdx.y;
    if (blockIdx.z)
        for_touched(c, blockIdx.x, [&](const Touched& b) { read_block<KT, DT, D, true>(c, b, h, v, ld_v, lds); });
    else
        for_touched(c, blockIdx.x, [&](const Touched& b) { read_block<KT, DT, D, false>(c, b, h, k, ld_k, lds); });
}

template <template <int, int, int> class L, class... A>
hipError_t by_type(readme_kv_type kt, readme_dtype dt, int D, A... a) {
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

dim3 kv_grid(const KvCacheArgs& c) {
    return dim3((unsigned)(c.R + ceil_div(c.T, kKvBlock)), (unsigned)c.Hk, 2u);
}

template <int KT, int DT, int D>
struct WriteOp {
    static hipError_t go(KvCacheArgs c, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                         hipStream_t s) {
        k_kv_write<KT, DT, D><<<kv_grid(c), kThreads, 0, s>>>(c, k, ld_k, v, ld_v);
        return hipGetLastError();
    }
};
template <int KT, int DT, int D>
struct ReadOp {
    static hipError_t go(KvCacheArgs c, void* k, int64_t ld_k, void* v, int64_t ld_v,
                         hipStream_t s) {
        k_kv_read<KT, DT, D><<<kv_grid(c), kThreads, 0, s>>>(c, k, ld_k, v, ld_v);
        return hipGetLastError();
    }
};

}  // namespace

hipError_t launch_kv_write(readme_kv_type kt, readme_dtype dt, const KvCacheArgs& c, const void* k,
                           int64_t ld_k, const void* v, int64_t ld_v, hipStream_t s) {
    return by_type<WriteOp>(kt, dt, c.D, c, k, ld_k, v, ld_v, s);
}

hipError_t launch_kv_read(readme_kv_type kt, readme_dtype dt, const KvCacheArgs& c, void* k,
                          int64_t ld_k, void* v, int64_t ld_v, hipStream_t s) {
    return by_type<ReadOp>(kt, dt, c.D, c, k, ld_k, v, ld_v, s);
}

}  // namespace readme
