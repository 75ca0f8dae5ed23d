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
#include "kv_write.hpp"

namespace readme {

namespace {

template <int KT, int DT, int D>
__global__ __launch_bounds__(kKvThreads) void k_kv_write(KvCacheArgs c, const void* __restrict__ k,
                                                         int64_t ld_k, const void* __restrict__ v,
                                                         int64_t ld_v) {
    write_candidate<KT, D>(c, false, PlainRows<DT>{k, ld_k}, PlainRows<DT>{v, ld_v});
}

template <int KT, int DT, int D, bool V>
__device__ __forceinline__ void read_block(const KvCacheArgs& c, const Touched& b, int h, void* out,
                                           int64_t ld, uint32_t* lds) {
    const int tid = threadIdx.x;
    constexpr int LPR = D / 16, RPP = kKvThreads / LPR, NP = kKvBlock / RPP;
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
            constexpr int NI = 2 * D / kKvThreads > 0 ? 2 * D / kKvThreads : 1;
            uint32_t in[NI][2][4];
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int i = tid + j * kKvThreads;
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
                const int i = tid + j * kKvThreads;
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
__global__ __launch_bounds__(kKvThreads) void k_kv_read(KvCacheArgs c, void* __restrict__ k, int64_t ld_k,
                                                      void* __restrict__ v, int64_t ld_v) {
    __shared__ uint32_t lds[kKvBlock * kv_lds_row(D)];
    const int h = blockIdx.y;
    if (blockIdx.z)
        for_touched(c, blockIdx.x, false, [&](const Touched& b) { read_block<KT, DT, D, true>(c, b, h, v, ld_v, lds); });
    else
        for_touched(c, blockIdx.x, false, [&](const Touched& b) { read_block<KT, DT, D, false>(c, b, h, k, ld_k, lds); });
}

template <int KT, int DT, int D>
struct WriteOp {
    static hipError_t go(KvCacheArgs c, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                         hipStream_t s) {
        k_kv_write<KT, DT, D><<<kv_grid(c), kKvThreads, 0, s>>>(c, k, ld_k, v, ld_v);
        return hipGetLastError();
    }
};
template <int KT, int DT, int D>
struct ReadOp {
    static hipError_t go(KvCacheArgs c, void* k, int64_t ld_k, void* v, int64_t ld_v,
                         hipStream_t s) {
        k_kv_read<KT, DT, D><<<kv_grid(c), kKvThreads, 0, s>>>(c, k, ld_k, v, ld_v);
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
