// C entry points of the 8-bit key/value cache and the attention over it: host
// checks, then the launches of kv_cache.hip and attention_kv_*.hip.
#include <limits.h>
#include <math.h>

#include "kv_cache.hpp"

using namespace readme;

namespace {

constexpr int64_t kMaxRequests = 1 << 22;
constexpr int64_t kMaxRows = 1 << 27;   // T H / Hk
// Tiles of 16 query rows times key heads: the attention grids, a workgroup of
// up to 256 threads for each, stay below 2^32 threads.
constexpr int64_t kMaxPairs = 1 << 23;
// Every position is below 2^31, and 2^27 rows may lie before the first: a window
// beyond this is none, and positions less it fit 64 bits.
constexpr int64_t kMaxWindow = 1ll << 33;

inline readme_status st_of(hipError_t e) { return e == hipSuccess ? README_OK : README_ERR_HIP; }
inline bool al(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }

bool head_dim_ok(int32_t D) { return D == 64 || D == 128 || D == 256; }

// Sizes first, so that a call of no rows asks for no pointers.  `done` is set
// where nothing is to be done.
readme_status check_sizes(readme_kv_type kt, int64_t T, int32_t R, int32_t H, int32_t Hk, int32_t D,
                          int64_t max_blocks, int64_t n_blocks, bool* done) {
    *done = false;
    if (T < 0 || R < 0 || H < 0 || Hk < 0 || max_blocks < 0 || n_blocks < 0) return README_ERR_ARG;
    if (kt != README_KV_I8 && kt != README_KV_E4M3) return README_ERR_UNSUPPORTED;
    if (!head_dim_ok(D) || Hk > 65535 || R > kMaxRequests) return README_ERR_UNSUPPORTED;
    if (max_blocks > INT32_MAX / kKvBlock || n_blocks > INT32_MAX) return README_ERR_UNSUPPORTED;
    if (T == 0) {
        *done = true;
        return README_OK;
    }
    if (R < 1 || Hk < 1 || H < 1 || max_blocks < 1 || n_blocks < 1) return README_ERR_ARG;
    if (H % Hk != 0) return README_ERR_ARG;
    if (T > kMaxRows / (H / Hk)) return README_ERR_UNSUPPORTED;
    return README_OK;
}

readme_status check_rows(const void* p, int64_t ld, int64_t width, int64_t elem) {
    if (!p || !al(p, 16) || ld < width || (ld * elem) % 16 != 0) return README_ERR_ARG;
    return README_OK;
}

}  // namespace

namespace readme {

readme_status kv_check_attention(readme_kv_type kt, int64_t T, int32_t R, int32_t H, int32_t Hk,
                                 int32_t D, int64_t max_blocks, int64_t n_blocks, bool* done) {
    const readme_status st = check_sizes(kt, T, R, H, Hk, D, max_blocks, n_blocks, done);
    if (st != README_OK || *done) return st;
    return (T * (H / Hk) / 16 + R) * Hk > kMaxPairs ? README_ERR_UNSUPPORTED : README_OK;
}

readme_status kv_check_cache(const KvCacheArgs& c) {
    if (!c.offsets || !c.lens || !c.table || !c.codes || !c.scales) return README_ERR_ARG;
    if (!al(c.offsets, 4) || !al(c.lens, 4) || !al(c.table, 4) || !al(c.codes, 16) ||
        !al(c.scales, 8))
        return README_ERR_ARG;
    return README_OK;
}

KvCacheArgs kv_cache_args(int64_t T, int32_t R, int32_t Hk, int32_t D, const int32_t* offsets,
                       const int32_t* lens, const int32_t* table, int64_t max_blocks,
                       int64_t n_blocks, const void* codes, const float* scales) {
    KvCacheArgs c{};
    c.T = T;
    c.R = R;
    c.Hk = Hk;
    c.D = D;
    c.offsets = offsets;
    c.lens = lens;
    c.table = table;
    c.max_blocks = max_blocks;
    c.n_blocks = n_blocks;
    c.codes = const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(codes));
    c.scales = const_cast<float*>(scales);
    return c;
}

}  // namespace readme

extern "C" {

size_t readme_kv_codes_bytes(int64_t n_blocks, int32_t Hk, int32_t D) {
    if (n_blocks < 0 || n_blocks > INT32_MAX || Hk < 1 || Hk > 65535 || !head_dim_ok(D)) return 0;
    return (size_t)n_blocks * Hk * 2 * kKvBlock * D;
}

size_t readme_kv_scales_bytes(int64_t n_blocks, int32_t Hk) {
    if (n_blocks < 0 || n_blocks > INT32_MAX || Hk < 1 || Hk > 65535) return 0;
    return (size_t)n_blocks * Hk * 2 * sizeof(float);
}

readme_status readme_kv_write(readme_kv_type kt, readme_dtype dt, int64_t T, int32_t R, int32_t Hk,
                              int32_t D, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                              const int32_t* offsets, const int32_t* lens, const int32_t* table,
                              int64_t max_blocks, int64_t n_blocks, void* codes, float* scales,
                              void* stream) {
    if (dt != README_F32 && dt != README_BF16) return README_ERR_UNSUPPORTED;
    bool done;
    readme_status st = check_sizes(kt, T, R, Hk, Hk, D, max_blocks, n_blocks, &done);
    if (st != README_OK || done) return st;
    const KvCacheArgs c = kv_cache_args(T, R, Hk, D, offsets, lens, table, max_blocks, n_blocks, codes,
                                     scales);
    if ((st = kv_check_cache(c)) != README_OK) return st;
    const int64_t es = (int64_t)dtype_size(dt), width = (int64_t)Hk * D;
    if ((st = check_rows(k, ld_k, width, es)) != README_OK) return st;
    if ((st = check_rows(v, ld_v, width, es)) != README_OK) return st;
    return st_of(launch_kv_write(kt, dt, c, k, ld_k, v, ld_v, as_stream(stream)));
}

readme_status readme_kv_read(readme_kv_type kt, readme_dtype dt, int64_t T, int32_t R, int32_t Hk,
                             int32_t D, const int32_t* offsets, const int32_t* lens,
                             const int32_t* table, int64_t max_blocks, int64_t n_blocks,
                             const void* codes, const float* scales, void* k, int64_t ld_k, void* v,
                             int64_t ld_v, void* stream) {
    if (dt != README_F32 && dt != README_BF16) return README_ERR_UNSUPPORTED;
    bool done;
    readme_status st = check_sizes(kt, T, R, Hk, Hk, D, max_blocks, n_blocks, &done);
    if (st != README_OK || done) return st;
    const KvCacheArgs c = kv_cache_args(T, R, Hk, D, offsets, lens, table, max_blocks, n_blocks, codes,
                                     scales);
    if ((st = kv_check_cache(c)) != README_OK) return st;
    const int64_t es = (int64_t)dtype_size(dt), width = (int64_t)Hk * D;
    if ((st = check_rows(k, ld_k, width, es)) != README_OK) return st;
    if ((st = check_rows(v, ld_v, width, es)) != README_OK) return st;
    return st_of(launch_kv_read(kt, dt, c, k, ld_k, v, ld_v, as_stream(stream)));
}

size_t readme_attention_kv_workspace_bytes(int64_t T, int32_t R, int32_t H, int32_t Hk, int32_t D,
                                           int64_t max_blocks) {
    bool done;
    if (kv_check_attention(README_KV_I8, T, R, H, Hk, D, max_blocks, 1, &done) != README_OK || done)
        return 0;
    return kv_attention_workspace(T, R, H, Hk, D, max_blocks);
}

readme_status readme_attention_kv(readme_kv_type kt, int64_t T, int32_t R, int32_t H, int32_t Hk,
                                  int32_t D, const void* q, int64_t ld_q, const int32_t* offsets,
                                  const int32_t* lens, const int32_t* table, int64_t max_blocks,
                                  int64_t n_blocks, const void* codes, const float* scales,
                                  float scale, int32_t causal, int64_t window, void* o,
                                  int64_t ld_o, void* workspace, size_t workspace_bytes,
                                  void* stream) {
    const float score = scale * 1.4426950408889634f;  // log2(e): weights are powers of two
    if (causal < 0 || causal > 1 || window < 0 || !(score > 0.0f) || !isfinite(score))
        return README_ERR_ARG;
    bool done;
    readme_status st = kv_check_attention(kt, T, R, H, Hk, D, max_blocks, n_blocks, &done);
    if (st != README_OK || done) return st;
    const KvCacheArgs c = kv_cache_args(T, R, Hk, D, offsets, lens, table, max_blocks, n_blocks, codes,
                                     scales);
    if ((st = kv_check_cache(c)) != README_OK) return st;
    const int64_t width = (int64_t)H * D;
    if ((st = check_rows(q, ld_q, width, 2)) != README_OK) return st;
    if ((st = check_rows(o, ld_o, width, 2)) != README_OK) return st;
    if (!workspace || !al(workspace, 16)) return README_ERR_ARG;
    if (workspace_bytes < kv_attention_workspace(T, R, H, Hk, D, max_blocks))
        return README_ERR_WORKSPACE;
    KvAttnArgs a{};
    a.c = c;
    a.q = reinterpret_cast<const uint16_t*>(q);
    a.ld_q = ld_q;
    a.o = reinterpret_cast<uint16_t*>(o);
    a.ld_o = ld_o;
    a.G = H / Hk;
    a.score = score;
    a.causal = causal;
    a.window = window < kMaxWindow ? window : kMaxWindow;
    a.ws = workspace;
    return st_of(launch_kv_attention(kt, a, as_stream(stream)));
}

}  // extern "C"
