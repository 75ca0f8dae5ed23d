// readme_kv_append: a call's keys, turned by their positions, and values into the
// 8-bit cache (rotary.hpp and kv_cache.hip have the mathematics).
//
// The write's own kernel with another source of K rows: a thread's sixteen dims
// are the two runs of eight whose pairs they make, so both members of a pair and
// its angle are in one thread and the turned fp32 values go from its registers into
// the codes.
// Bound by instructions: 16155 rows of 8 heads of 128, bf16 to e4m3, 99 MB, in 39 us
// with the angles anew for every head, vector ALU at work in 76% of the busy cycles, and
// in 32.5 with sines and cosines shared by four heads, through LDS (69%; through
// registers, 165 of them, 39 to 45); the write alone 29.  K's workgroups come before
// V's, which are the shorter: in turns 43 for the 39.  A row each of 64 requests 6.6, the
// launch and four dependent loads.
#include "kv_write.hpp"

namespace readme {

namespace {

__device__ __forceinline__ Row16<README_F32> turned_row(const float (&v)[16]) {
    Row16<README_F32> o;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        o.v[i] = make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]),
                            __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
    return o;
}
// The position that a row turns by; a stored one fits 32 bits unless its block is absent.
__device__ __forceinline__ int position_of(const RotaryArgs& rot, const Touched& b, int row) {
    return rot.pos ? rot.pos[b.tok + row] : (int)(b.j * kKvBlock + b.slot + row);
}

// The call's key rows, turned.  The angles' frequencies and the row's position are
// on their way with the row.
template <int DT>
struct TurnedRows {
    static constexpr int kType = README_F32;
    static constexpr bool kOneRun = false;
    static constexpr int N = DT == README_F32 ? 2 : 1;
    struct Raw {
        uint4 a[N], b[N];
        int pos;
    };
    const void* base;
    int64_t ld;
    RotaryArgs rot;
    double f[8];  // of the thread's pairs

    __device__ __forceinline__ TurnedRows(const void* k, int64_t ld_k, const RotaryArgs& r, int ch)
        : base(k), ld(ld_k), rot(r) {
        if (chunk(ch).turns) {
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = rot.freqs[8 * ch + e];
        }
    }
    __device__ __forceinline__ Chunk chunk(int ch) const { return chunk_of(ch, rot.rot, rot.layout); }
    __device__ __forceinline__ void zero(Raw& x) const {
#pragma unroll
        for (int i = 0; i < N; ++i) x.a[i] = x.b[i] = make_uint4(0u, 0u, 0u, 0u);
        x.pos = 0;
    }
    __device__ __forceinline__ void load(Raw& x, const Touched& b, int row, int col, int ch) const {
        const Chunk k = chunk(ch);
        const int64_t at = (b.tok + row) * ld + col;
        load8<DT>(base, at + k.a, x.a);
        load8<DT>(base, at + k.b, x.b);
        x.pos = position_of(rot, b, row);
    }
    // Row `row` of the block's rows; zeros past the last.
    __device__ __forceinline__ Row16<README_F32> value(const Raw& x, const Touched& b, int row, int ch) const {
        float v[16];
        widen8<DT>(x.a, v);
        widen8<DT>(x.b, v + 8);
        if (chunk(ch).turns && row < b.n) {
            Turn t[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) t[e] = turn_of((double)x.pos, f[e], rot.amplitude, 1.0f);
            turn_chunk(t, rot.layout, v);
        }
        return turned_row(v);
    }
};

// The same with a block's sines and cosines kept for all the heads that a workgroup
// writes, in LDS, where a thread reads what it wrote itself.
template <int DT, int D>
struct KeptRows {
    static constexpr int kType = README_F32;
    static constexpr bool kOneRun = false;
    static constexpr int N = DT == README_F32 ? 2 : 1;
    static constexpr int kItems = kKvBlock * (D / 16);  // a block's chunks
    struct Raw {
        uint4 a[N], b[N];
    };
    const void* base;
    int64_t ld;
    RotaryArgs rot;
    float4* kept;  // [4][kItems], two pairs each

    __device__ __forceinline__ Chunk chunk(int ch) const { return chunk_of(ch, rot.rot, rot.layout); }
    __device__ __forceinline__ void keep(const Touched& b) const {
        const int ch = threadIdx.x % (D / 16);
        if (!chunk(ch).turns) return;
        double f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = rot.freqs[8 * ch + e];
#pragma unroll
        for (int i = threadIdx.x; i < kItems; i += kKvThreads) {
            const int row = i / (D / 16);
            if (row >= b.n) break;
            const double pos = (double)position_of(rot, b, row);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const Turn t = turn_of(pos, f[2 * k], rot.amplitude, 1.0f);
                const Turn u = turn_of(pos, f[2 * k + 1], rot.amplitude, 1.0f);
                kept[k * kItems + i] = make_float4(t.c, t.s, u.c, u.s);
            }
        }
    }
    __device__ __forceinline__ void zero(Raw& x) const {
#pragma unroll
        for (int i = 0; i < N; ++i) x.a[i] = x.b[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ __forceinline__ void load(Raw& x, const Touched& b, int row, int col, int ch) const {
        const Chunk k = chunk(ch);
        const int64_t at = (b.tok + row) * ld + col;
        load8<DT>(base, at + k.a, x.a);
        load8<DT>(base, at + k.b, x.b);
    }
    __device__ __forceinline__ Row16<README_F32> value(const Raw& x, const Touched& b, int row, int ch) const {
        float v[16];
        widen8<DT>(x.a, v);
        widen8<DT>(x.b, v + 8);
        if (chunk(ch).turns && row < b.n) {
            Turn t[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float4 c = kept[k * kItems + row * (D / 16) + ch];
                t[2 * k] = Turn{c.x, c.y};
                t[2 * k + 1] = Turn{c.z, c.w};
            }
            turn_chunk(t, rot.layout, v);
        }
        return turned_row(v);
    }
};

template <int KT, int DT, int D>
__global__ __launch_bounds__(kKvThreads) void k_kv_append(KvCacheArgs c, RotaryArgs rot, bool apart,
                                                          const void* __restrict__ k, int64_t ld_k,
                                                          const void* __restrict__ v, int64_t ld_v) {
    write_candidate<KT, D>(c, apart, TurnedRows<DT>(k, ld_k, rot, threadIdx.x % (D / 16)),
                           PlainRows<DT>{v, ld_v});
}

// Of many rows: K of kHeads heads to a workgroup, blockIdx.y < groups, then V of one.
// Held to 128 registers, four workgroups to a CU: with 138, three, 36 for the 32.5.
constexpr int kHeads = 4;
template <int KT, int DT, int D>
__global__ __launch_bounds__(kKvThreads, 4) void k_kv_append_heads(KvCacheArgs c, RotaryArgs rot, int groups,
                                                                const void* __restrict__ k, int64_t ld_k,
                                                                const void* __restrict__ v, int64_t ld_v) {
    __shared__ uint32_t most[4];
    __shared__ __attribute__((aligned(16))) uint32_t lds[KeptRows<DT, D>::kItems * 16];
    static_assert(KeptRows<DT, D>::kItems * 16 >= kKvBlock * kv_lds_row(D), "V's codes fit too");
    const int y = blockIdx.y;
    if (y >= groups) {
        for_touched(c, blockIdx.x, false, [&](const Touched& b) {
            write_block<KT, D, true>(c, b, y - groups, PlainRows<DT>{v, ld_v}, lds, most);
        });
    } else {
        const KeptRows<DT, D> rows{k, ld_k, rot, reinterpret_cast<float4*>(lds)};
        for_touched(c, blockIdx.x, false, [&](const Touched& b) {
            rows.keep(b);
            for (int h = y * kHeads; h < c.Hk && h < (y + 1) * kHeads; ++h)
                write_block<KT, D, false>(c, b, h, rows, lds, most);
        });
    }
}

// Whether second blocks are candidates of their own.  R Hk 2 workgroups more, most of
// them with nothing to do, against up to 32 blocks one after the other: 17 requests of
// 5 to 33 rows, 3 heads, 7 us for 14; 300 of 2 rows, 8 heads, 28 for 13.
bool second_apart(const KvCacheArgs& c) { return c.T > c.R && c.R * c.Hk <= 256; }

// Whether four heads share a workgroup, from three units of 64 rows and a head to a CU:
// us, shared against not (e4m3, heads of 128): 16155 rows of 8 heads 32.5 for 39.8, 8200
// of 32 59 for 73, 4096 of 16 20.2 for 22.7, 400 requests of 30 rows 55 for 64, 8 of 768,
// three units, 18.8 for 19.1; 4096 rows of 8 17.7 for 15.8, 3000 of 8 15.9 for 9.8.  Heads
// of 64: 25 for 31, at three units 14.6 for 15.9.  A row each of 8192 requests, 8 heads,
// 404 for 467.  Of 256, whose sines and cosines are 64 KB: 8192 rows of 8 heads 38.5 and
// 39.6 (int8, e4m3) for 41.3 and 41.4, 16160 of 8 66.5 and 71.4 for 68.5 and 71.8, 8192
// of 4 27 and 29 for 24: not worth the kernels.
bool heads_share(const KvCacheArgs& c) {
    return c.Hk > 1 && c.Hk <= 32768 && c.T * c.Hk >= 3 * 256 * kKvBlock;  // blockIdx.y below 2^16
}

enum Form : int { kOneByOne, kSecondApart, kHeadsShare };
Form form_of(const KvCacheArgs& c) {
    if (c.D < 256 && heads_share(c)) return kHeadsShare;
    return second_apart(c) ? kSecondApart : kOneByOne;
}

template <int KT, int DT, int D>
struct AppendOp {
    static hipError_t go(KvCacheArgs c, RotaryArgs rot, const void* k, int64_t ld_k, const void* v,
                         int64_t ld_v, hipStream_t s) {
        const Form form = form_of(c);
        if constexpr (D < 256) {
            if (form == kHeadsShare) {
                const int groups = (c.Hk + kHeads - 1) / kHeads;
                const dim3 grid(kv_grid(c).x, (unsigned)(groups + c.Hk));
                k_kv_append_heads<KT, DT, D><<<grid, kKvThreads, 0, s>>>(c, rot, groups, k, ld_k, v, ld_v);
                return hipGetLastError();
            }
        }
        dim3 grid = kv_grid(c);
        if (form == kSecondApart) grid.x += (unsigned)c.R;
        k_kv_append<KT, DT, D><<<grid, kKvThreads, 0, s>>>(c, rot, form == kSecondApart, k, ld_k, v, ld_v);
        return hipGetLastError();
    }
};

}  // namespace

hipError_t launch_kv_append(readme_kv_type kt, readme_dtype dt, const KvCacheArgs& c,
                            const RotaryArgs& rot, const void* k, int64_t ld_k, const void* v,
                            int64_t ld_v, hipStream_t s) {
    return by_type<AppendOp>(kt, dt, c.D, c, rot, k, ld_k, v, ld_v, s);
}

}  // namespace readme

// For the tests: how a call's blocks and heads are dealt to workgroups, 0 one by one, 1
// second blocks apart, 2 heads sharing sines and cosines.
extern "C" int32_t readme_internal_kv_append_form(int64_t T, int32_t R, int32_t Hk, int32_t D) {
    readme::KvCacheArgs c{};
    c.T = T;
    c.R = R;
    c.Hk = Hk;
    c.D = D;
    return readme::form_of(c);
}
