// readme_kv_append: a call's keys, turned by their positions, and values into the
// 8-bit cache (rotary.hpp and kv_cache.hip have the mathematics).
//
// The write's own kernel with another source of K rows: a thread's sixteen dims
// are the two runs of eight whose pairs they make, so both members of a pair and
// its angle are in one thread and the turned fp32 values go from its registers into
// the codes.
// Each head turns its own rows by angles that all heads share: sines and cosines
// once for two or four heads need 165 registers instead of 124, and 39 to 45 us where
// this takes 39 (16155 rows of 8 heads of 128, bf16 to e4m3, 99 MB; the write alone 29,
// the turn's instructions the rest: vector ALU at work in 76% of the busy cycles).  K's
// workgroups come before V's, which are the shorter: in turns 43.  A row each of 64
// requests 6.6, the launch and four dependent loads.
#include "kv_write.hpp"

namespace readme {

namespace {

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
        // A stored position fits 32 bits unless its block is absent
        x.pos = rot.pos ? rot.pos[b.tok + row] : (int)(b.j * kKvBlock + b.slot + row);
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
        Row16<README_F32> o;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            o.v[i] = make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]),
                                __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
        return o;
    }
};

template <int KT, int DT, int D>
__global__ __launch_bounds__(kKvThreads) void k_kv_append(KvCacheArgs c, RotaryArgs rot, bool apart,
                                                          const void* __restrict__ k, int64_t ld_k,
                                                          const void* __restrict__ v, int64_t ld_v) {
    write_candidate<KT, D>(c, apart, TurnedRows<DT>(k, ld_k, rot, threadIdx.x % (D / 16)),
                           PlainRows<DT>{v, ld_v});
}

// Whether second blocks are candidates of their own.  R Hk 2 workgroups more, most of
// them with nothing to do, against up to 32 blocks one after the other: 17 requests of
// 5 to 33 rows, 3 heads, 7 us for 14; 300 of 2 rows, 8 heads, 28 for 13.
bool second_apart(const KvCacheArgs& c) { return c.T > c.R && c.R * c.Hk <= 256; }

template <int KT, int DT, int D>
struct AppendOp {
    static hipError_t go(KvCacheArgs c, RotaryArgs rot, const void* k, int64_t ld_k, const void* v,
                         int64_t ld_v, hipStream_t s) {
        const bool apart = second_apart(c);
        dim3 grid = kv_grid(c);
        if (apart) grid.x += (unsigned)c.R;
        k_kv_append<KT, DT, D><<<grid, kKvThreads, 0, s>>>(c, rot, apart, k, ld_k, v, ld_v);
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
