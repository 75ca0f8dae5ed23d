// The 8-bit key/value cache (readme_kv_*): its layout, its codes and how a
// call's rows are found in it.  Shared by kv_cache.hip (write, read) and
// attention_kv*.hip.
//
// A block is 64 tokens of one request.  Per block and key/value head:
//   K codes  [2][D / 16][32][16]  token half, 16-dim chunk, token, dim
//   V codes  [2][D][32]           token half, dim, token
// so that the sixteen bytes a lane loads are one operand row of the matrix
// cores in either product: 16 dims of one key for Q K^T (summed over dims), 16
// tokens of one dim for P V (summed over tokens), and neighbouring lanes read
// neighbouring pieces.
#pragma once

#include "common.hpp"
#include "internal.hpp"

namespace readme {

constexpr int kKvBlock = 64;
// Scales are at least this: a block of zeros has no scale of its own, and a
// reciprocal stays finite.
constexpr float kKvScaleFloor = 7.888609052210118e-31f;  // 2^-100

template <int KT>
constexpr float kv_qmax() {
    return KT == README_KV_I8 ? 127.0f : 448.0f;
}

// Bytes of one (block, head)'s K or V codes.
__device__ __forceinline__ int64_t kv_half_bytes(int D) { return (int64_t)kKvBlock * D; }
// Byte of (token slot, dim) in a (block, head)'s K codes and V codes.
__device__ __forceinline__ int kv_k_byte(int D, int slot, int d) {
    return (((slot >> 5) * (D >> 4) + (d >> 4)) * 32 + (slot & 31)) * 16 + (d & 15);
}
__device__ __forceinline__ int kv_v_byte(int D, int slot, int d) {
    return ((slot >> 5) * D + d) * 32 + (slot & 31);
}

// Pool block of a request's block j, or -1 where the request has none there.
__device__ __forceinline__ int64_t kv_block_of(const int32_t* __restrict__ table,
                                               int64_t max_blocks, int64_t n_blocks, int64_t r,
                                               int64_t j) {
    if (j < 0 || j >= max_blocks) return -1;
    const int64_t b = table[r * max_blocks + j];
    return b >= 0 && b < n_blocks ? b : -1;
}

// Rows [lo, hi) of request r, kept inside [0, T] whatever the offsets hold.
__device__ __forceinline__ void kv_clamp_rows(int64_t a, int64_t b, int64_t T, int64_t& lo,
                                              int64_t& hi) {
    lo = a < 0 ? 0 : (a > T ? T : a);
    hi = b < lo ? lo : (b > T ? T : b);
}
__device__ __forceinline__ void kv_rows(const int32_t* __restrict__ offsets, int64_t T, int64_t r,
                                        int64_t& lo, int64_t& hi) {
    kv_clamp_rows(offsets[r], offsets[r + 1], T, lo, hi);
}

// The last request r with offsets[r] <= t (0 if none), found by the 64 lanes
// of a wave together: each step reads 64 evenly spaced offsets.
__device__ __forceinline__ int64_t kv_request_at(const int32_t* __restrict__ offsets, int64_t R,
                                                 int64_t t) {
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, n = R;
    while (n > 1) {
        const int64_t step = (n + 63) / 64;
        const int64_t i = lane * step;
        const bool le = i < n && offsets[lo + i] <= t;
        const int below = __popcll(__ballot(le));
        const int64_t skip = below > 0 ? (int64_t)(below - 1) * step : 0;
        lo += skip;
        n = n - skip < step ? n - skip : step;
    }
    return lo;
}

// floor(a / 64) and a mod 64 for any sign.
__device__ __forceinline__ int64_t kv_block_index(int64_t p) { return p >> 6; }
__device__ __forceinline__ int kv_slot(int64_t p) { return (int)(p & 63); }

// Arguments of a cache as the kernels take them.
struct KvCacheArgs {
    int64_t T;
    int64_t R;
    const int32_t* offsets;
    const int32_t* lens;
    const int32_t* table;
    int64_t max_blocks, n_blocks;
    uint8_t* codes;
    float* scales;
    int Hk, D;
};

// The host checks of the entry points (kv_abi.hip), sizes before pointers.
// `done`: there are no rows.
readme_status kv_check_attention(readme_kv_type kt, int64_t T, int32_t R, int32_t H, int32_t Hk,
                                 int32_t D, int64_t max_blocks, int64_t n_blocks, bool* done);
readme_status kv_check_cache(const KvCacheArgs& c);
KvCacheArgs kv_cache_args(int64_t T, int32_t R, int32_t Hk, int32_t D, const int32_t* offsets,
                          const int32_t* lens, const int32_t* table, int64_t max_blocks,
                          int64_t n_blocks, const void* codes, const float* scales);

hipError_t launch_kv_write(readme_kv_type kt, readme_dtype dt, const KvCacheArgs& c, const void* k,
                           int64_t ld_k, const void* v, int64_t ld_v, hipStream_t s);
struct RotaryArgs;
hipError_t launch_kv_append(readme_kv_type kt, readme_dtype dt, const KvCacheArgs& c,
                            const RotaryArgs& rot, const void* k, int64_t ld_k, const void* v,
                            int64_t ld_v, hipStream_t s);
hipError_t launch_kv_read(readme_kv_type kt, readme_dtype dt, const KvCacheArgs& c, void* k,
                          int64_t ld_k, void* v, int64_t ld_v, hipStream_t s);

// Attention over a cache (attention_kv.hip).
struct KvAttnArgs {
    KvCacheArgs c;
    const uint16_t* q;
    int64_t ld_q;
    uint16_t* o;
    int64_t ld_o;
    int G;            // query heads per key/value head
    float score;      // log2(e) * softmax scale
    int causal;
    int64_t window;   // 0: none
    // Rows of a draft tree, else NULL: who sees whom, and the rows' positions
    // (NULL: those they are stored at).
    const uint64_t* tree;
    int64_t words;
    const int32_t* pos;
    void* ws;
};
size_t kv_attention_workspace(bool tree, int64_t T, int64_t R, int H, int Hk, int D, int64_t max_blocks);
hipError_t launch_kv_attention(readme_kv_type kt, const KvAttnArgs& a, hipStream_t s);

}  // namespace readme
