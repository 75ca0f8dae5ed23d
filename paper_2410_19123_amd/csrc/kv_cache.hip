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
// one wave per (candidate, head, K or V) and need no plan and no workspace.
#include <math.h>

#include "kv_cache.hpp"

namespace readme {

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

// 16 consecutive values of a row in fp32.
template <int DT>
__device__ __forceinline__ void load16(const void* base, int64_t at, float (&x)[16]) {
    if constexpr (DT == README_BF16) {
        const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(base) + at);
        const uint4 a = p[0], b = p[1];
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[2 * i] = bf16_lo(w[i]);
            x[2 * i + 1] = bf16_hi(w[i]);
        }
    } else {
        const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(base) + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 a = p[i];
            x[4 * i] = a.x;
            x[4 * i + 1] = a.y;
            x[4 * i + 2] = a.z;
            x[4 * i + 3] = a.w;
        }
    }
}

template <int DT>
__device__ __forceinline__ void store16(void* base, int64_t at, const float (&x)[16]) {
    if constexpr (DT == README_BF16) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            w[i] = (uint32_t)f32_to_bf16(x[2 * i]) | ((uint32_t)f32_to_bf16(x[2 * i + 1]) << 16);
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

// The code byte nearest to x / s (inv = 1 / s in fp32), ties to even.
//   int8: n = rint(x * inv) is at most one off; x - n s is exact in fp32 (a
//   multiple of s's last place and at most 1.5 s, or x near s), so comparing
//   it with s / 2 settles n.
//   e4m3: one Newton step makes q faithful (less than one unit off), the sign
//   of x - q s tells on which side x / s lies, and taking the neighbour with
//   an odd last bit (round to odd) keeps the hardware's second rounding from
//   seeing a tie where there is none.
template <int KT>
__device__ __forceinline__ uint32_t encode(float x, float s, float inv) {
    if constexpr (KT == README_KV_I8) {
        float n = rintf(x * inv);
        const float r = fmaf(-n, s, x), h = 0.5f * s;
        const bool odd = ((int)n & 1) != 0;
        if (r > h || (r == h && odd)) n += 1.0f;
        else if (r < -h || (r == -h && odd)) n -= 1.0f;
        n = fminf(fmaxf(n, -127.0f), 127.0f);
        return (uint32_t)((int)n + 128);
    } else {
        float q = x * inv;
        q = fmaf(fmaf(-q, s, x), inv, q);
        const float r = fmaf(-q, s, x);
        uint32_t u = __float_as_uint(q);
        if (r != 0.0f && !(u & 1u)) u = ((r > 0.0f) == (q > 0.0f)) ? u + 1u : u - 1u;
        if (q == 0.0f) u = 0u;
        return e4m3_byte(fminf(fmaxf(__uint_as_float(u), -448.0f), 448.0f));
    }
}

// The value a code stands for, and the code nearest to a value on the grid's
// own scale (ties to even).
template <int KT>
__device__ __forceinline__ float decode(uint32_t b) {
    if constexpr (KT == README_KV_I8) return (float)((int)b - 128);
    return __builtin_amdgcn_cvt_f32_fp8((int)b, 0);
}
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

// LDS bytes of one V wave: 64 token rows of D codes, four bytes apart per row
// so that a column's bytes spread over the banks.
constexpr int kv_lds_row(int D) { return D + 4; }

// One wave's block of K (half 0) or V (half 1).
template <int KT, int DT, int D, bool V>
__device__ __forceinline__ void write_block(const KvCacheArgs& c, const Touched& b, int h,
                                            const void* src, int64_t ld, uint8_t* lds) {
    const int64_t blk = kv_block_of(c.table, c.max_blocks, c.n_blocks, b.r, b.j);
    if (blk < 0) return;
    const int lane = threadIdx.x & 63;
    constexpr int LPR = D / 16;      // lanes per row, 16 values each
    constexpr int RPP = 64 / LPR;    // rows per pass
    const int ch = lane % LPR, rw = lane / LPR;
    const int64_t unit = (blk * c.Hk + h) * 2 + (V ? 1 : 0);
    uint8_t* dst = c.codes + unit * kv_half_bytes(D);
    const int64_t col = (int64_t)h * D + ch * 16;

    uint32_t am = 0;
    for (int i = rw; i < b.n; i += RPP) {
        float x[16];
        load16<DT>(src, (b.tok + i) * ld + col, x);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const uint32_t u = __float_as_uint(x[k]) & 0x7fffffffu;
            am = u > am ? u : am;
        }
    }
    am = wave_max_u32(am);
    const float need = __uint_as_float(am) / kv_qmax<KT>();
    float s = fmaxf(need, kKvScaleFloor), shrink = 1.0f;
    bool bad = am >= 0x7f800000u;
    if (b.slot > 0) {
        const float old = c.scales[unit];
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
    if (lane == 0) c.scales[unit] = s;
    const float inv = 1.0f / s;
    const uint32_t zero = KT == README_KV_I8 ? 0x80808080u : 0u;

    if constexpr (!V) {
        if (grown) {
            for (int i = lane; i < b.slot * LPR; i += 64) {
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
    const bool staged = V && (grown || b.n > RPP);
    for (int i = rw; i < b.n; i += RPP) {
        uint32_t w[4] = {zero, zero, zero, zero};
        if (!bad) {
            float x[16];
            load16<DT>(src, (b.tok + i) * ld + col, x);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                w[k] = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[k] |= encode<KT>(x[4 * k + e], s, inv) << (8 * e);
            }
        }
        if constexpr (!V) {
            *reinterpret_cast<uint4*>(dst + kv_k_byte(D, b.slot + i, ch * 16)) =
                make_uint4(w[0], w[1], w[2], w[3]);
        } else if (staged) {
            uint32_t* row = reinterpret_cast<uint32_t*>(lds + (b.slot + i) * kv_lds_row(D) + ch * 16);
#pragma unroll
            for (int k = 0; k < 4; ++k) row[k] = w[k];
        } else {
#pragma unroll
            for (int k = 0; k < 16; ++k)
                dst[kv_v_byte(D, b.slot + i, ch * 16 + k)] = (uint8_t)(w[k >> 2] >> (8 * (k & 3)));
        }
    }
    if constexpr (V) {
        if (!staged) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        // 16 tokens of one dim at a time: the new bytes from LDS, the earlier
        // ones rescaled, later ones left as they were.
        const int end = b.slot + b.n;
        for (int i = lane; i < 4 * D; i += 64) {
            const int d = i >> 1 & (D - 1), t0 = (i / (2 * D)) * 32 + (i & 1) * 16;
            if (t0 >= end || (t0 + 16 <= b.slot && !grown)) continue;
            uint4* p = reinterpret_cast<uint4*>(dst + kv_v_byte(D, t0, d));
            uint4 old = make_uint4(0u, 0u, 0u, 0u);
            if (t0 < b.slot || t0 + 16 > end) old = *p;
            uint32_t w[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int t = t0 + k, sh = 8 * (k & 3);
                uint32_t byte = (w[k >> 2] >> sh) & 0xffu;
                if (t >= b.slot && t < end) byte = lds[t * kv_lds_row(D) + d];
                else if (t < b.slot && grown) byte = regrid<KT>(byte, shrink);
                w[k >> 2] = (w[k >> 2] & ~(0xffu << sh)) | (byte << sh);
            }
            *p = make_uint4(w[0], w[1], w[2], w[3]);
        }
        // The next block of this wave writes the same LDS rows.
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// Two waves: K and V of (candidate blockIdx.x, head blockIdx.y).
template <int KT, int DT, int D>
__global__ __launch_bounds__(128) void k_kv_write(KvCacheArgs c, const void* __restrict__ k,
                                                  int64_t ld_k, const void* __restrict__ v,
                                                  int64_t ld_v) {
    __shared__ uint8_t lds[kKvBlock * kv_lds_row(D)];
    const int h = blockIdx.y;
    const bool isv = threadIdx.x >= 64;
    for_touched(c, blockIdx.x, [&](const Touched& b) {
        if (isv) write_block<KT, DT, D, true>(c, b, h, v, ld_v, lds);
        else write_block<KT, DT, D, false>(c, b, h, k, ld_k, lds);
    });
}

template <int KT, int DT, int D, bool V>
__device__ __forceinline__ void read_block(const KvCacheArgs& c, const Touched& b, int h, void* out,
                                           int64_t ld, uint8_t* lds) {
    const int lane = threadIdx.x & 63;
    constexpr int LPR = D / 16, RPP = 64 / LPR;
    const int ch = lane % LPR, rw = lane / LPR;
    const int64_t blk = kv_block_of(c.table, c.max_blocks, c.n_blocks, b.r, b.j);
    const int64_t unit = blk < 0 ? 0 : (blk * c.Hk + h) * 2 + (V ? 1 : 0);
    const uint8_t* src = c.codes + unit * kv_half_bytes(D);
    const float s = blk < 0 ? 0.0f : c.scales[unit];
    const int64_t col = (int64_t)h * D + ch * 16;
    if constexpr (V) {
        if (blk >= 0) {
            for (int i = lane; i < 4 * D; i += 64) {
                const int d = i >> 1 & (D - 1), t0 = (i / (2 * D)) * 32 + (i & 1) * 16;
                if (t0 >= b.slot + b.n || t0 + 16 <= b.slot) continue;
                const uint4 w = *reinterpret_cast<const uint4*>(src + kv_v_byte(D, t0, d));
                const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int k = 0; k < 16; ++k)
                    lds[(t0 + k) * kv_lds_row(D) + d] = (uint8_t)(ws[k >> 2] >> (8 * (k & 3)));
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    for (int i = rw; i < b.n; i += RPP) {
        float x[16];
        if (blk < 0) {
#pragma unroll
            for (int k = 0; k < 16; ++k) x[k] = 0.0f;
        } else {
            uint32_t w[4];
            if constexpr (V) {
                const uint32_t* row =
                    reinterpret_cast<const uint32_t*>(lds + (b.slot + i) * kv_lds_row(D) + ch * 16);
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = row[k];
            } else {
                const uint4 a =
                    *reinterpret_cast<const uint4*>(src + kv_k_byte(D, b.slot + i, ch * 16));
                w[0] = a.x;
                w[1] = a.y;
                w[2] = a.z;
                w[3] = a.w;
            }
#pragma unroll
            for (int k = 0; k < 16; ++k) x[k] = decode<KT>((w[k >> 2] >> (8 * (k & 3))) & 0xffu) * s;
        }
        store16<DT>(out, (b.tok + i) * ld + col, x);
    }
    if constexpr (V) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

template <int KT, int DT, int D>
__global__ __launch_bounds__(128) void k_kv_read(KvCacheArgs c, void* __restrict__ k, int64_t ld_k,
                                                 void* __restrict__ v, int64_t ld_v) {
    __shared__ uint8_t lds[kKvBlock * kv_lds_row(D)];
    const int h = blockIdx.y;
    const bool isv = threadIdx.x >= 64;
    for_touched(c, blockIdx.x, [&](const Touched& b) {
        if (isv) read_block<KT, DT, D, true>(c, b, h, v, ld_v, lds);
        else read_block<KT, DT, D, false>(c, b, h, k, ld_k, lds);
    });
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
    return dim3((unsigned)(c.R + ceil_div(c.T, kKvBlock)), (unsigned)c.Hk);
}

template <int KT, int DT, int D>
struct WriteOp {
    static hipError_t go(KvCacheArgs c, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                         hipStream_t s) {
        k_kv_write<KT, DT, D><<<kv_grid(c), 128, 0, s>>>(c, k, ld_k, v, ld_v);
        return hipGetLastError();
    }
};
template <int KT, int DT, int D>
struct ReadOp {
    static hipError_t go(KvCacheArgs c, void* k, int64_t ld_k, void* v, int64_t ld_v,
                         hipStream_t s) {
        k_kv_read<KT, DT, D><<<kv_grid(c), 128, 0, s>>>(c, k, ld_k, v, ld_v);
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
