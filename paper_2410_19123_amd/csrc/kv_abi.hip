// C entry points of the 8-bit key/value cache and the attention over it: host
// checks, then the launches of kv_cache.hip and attention_kv_*.hip.
#include <limits.h>
#include <math.h>

#include "kv_cache.hpp"
#include "rotary.hpp"

using namespace readme;

namespace {

constexpr int64_t kMaxRequests = 1 << 22;
constexpr int64_t kMaxRows = 1 << 27;   // T H / Hk
// Tiles of 16 query rows times key heads: the attention grids, a workgroup of
// up to 256 threads for each (of 512 where few run), stay below 2^32 threads.
constexpr int64_t kMaxPairs = 1 << 23;
// Every position is below 2^31, and 2^27 rows may lie before the first: a window
// beyond this is none, and positions less it fit 64 bits.
constexpr int64_t kMaxWindow = 1ll << 33;

inline readme_status st_of(hipError_t e) { return e == hipSuccess ? README_OK : README_ERR_HIP; }
inline bool al(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }

constexpr float kLog2e = 1.4426950408889634f;  // weights are powers of two
constexpr int32_t kMaxWords = 65536;           // of a row's bits in a draft tree

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

namespace {

// Checks of both attention calls, and what their kernels take alike.
readme_status attention_args(readme_kv_type kt, int64_t T, int32_t R, int32_t H, int32_t Hk,
                             int32_t D, const void* q, int64_t ld_q, const int32_t* offsets,
                             const int32_t* lens, const int32_t* table, int64_t max_blocks,
                             int64_t n_blocks, const void* codes, const float* scales, float score,
                             int64_t window, void* o, int64_t ld_o, bool tree, void* workspace,
                             size_t workspace_bytes, KvAttnArgs* a, bool* done) {
    readme_status st = kv_check_attention(kt, T, R, H, Hk, D, max_blocks, n_blocks, done);
    if (st != README_OK || *done) return st;
    a->c = kv_cache_args(T, R, Hk, D, offsets, lens, table, max_blocks, n_blocks, codes, scales);
    if ((st = kv_check_cache(a->c)) != README_OK) return st;
    const int64_t width = (int64_t)H * D;
    if ((st = check_rows(q, ld_q, width, 2)) != README_OK) return st;
    if ((st = check_rows(o, ld_o, width, 2)) != README_OK) return st;
    if (!workspace || !al(workspace, 16)) return README_ERR_ARG;
    if (workspace_bytes < kv_attention_workspace(tree, T, R, H, Hk, D, max_blocks))
        return README_ERR_WORKSPACE;
    a->q = reinterpret_cast<const uint16_t*>(q);
    a->ld_q = ld_q;
    a->o = reinterpret_cast<uint16_t*>(o);
    a->ld_o = ld_o;
    a->G = H / Hk;
    a->score = score;
    a->window = window < kMaxWindow ? window : kMaxWindow;
    a->ws = workspace;
    return README_OK;
}

}  // namespace

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

readme_status readme_kv_append(readme_kv_type kt, readme_dtype dt, int64_t T, int32_t R, int32_t Hk,
                               int32_t D, int32_t rot, readme_rotary_layout layout,
                               float amplitude, const int32_t* pos, const double* freqs,
                               const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                               const int32_t* offsets, const int32_t* lens, const int32_t* table,
                               int64_t max_blocks, int64_t n_blocks, void* codes, float* scales,
                               void* stream) {
    if (dt != README_F32 && dt != README_BF16) return README_ERR_UNSUPPORTED;
    bool done;
    readme_status st = check_sizes(kt, T, R, Hk, Hk, D, max_blocks, n_blocks, &done);
    if (st != README_OK) return st;
    if ((st = rotary_check_sizes(D, rot, layout, 0, amplitude)) != README_OK || done) return st;
    const KvCacheArgs c = kv_cache_args(T, R, Hk, D, offsets, lens, table, max_blocks, n_blocks, codes,
                                     scales);
    if ((st = kv_check_cache(c)) != README_OK) return st;
    if (!freqs || !al(freqs, 8) || !al(pos, 4)) return README_ERR_ARG;
    const int64_t es = (int64_t)dtype_size(dt), width = (int64_t)Hk * D;
    if ((st = check_rows(k, ld_k, width, es)) != README_OK) return st;
    if ((st = check_rows(v, ld_v, width, es)) != README_OK) return st;
    RotaryArgs a;
    a.pos = pos;
    a.freqs = freqs;
    a.amplitude = amplitude;
    a.rot = rot;
    a.layout = layout;
    a.inverse = 0;
    return st_of(launch_kv_append(kt, dt, c, a, k, ld_k, v, ld_v, as_stream(stream)));
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
    return kv_attention_workspace(false, T, R, H, Hk, D, max_blocks);
}

readme_status readme_attention_kv(readme_kv_type kt, int64_t T, int32_t R, int32_t H, int32_t Hk,
                                  int32_t D, const void* q, int64_t ld_q, const int32_t* offsets,
                                  const int32_t* lens, const int32_t* table, int64_t max_blocks,
                                  int64_t n_blocks, const void* codes, const float* scales,
                                  float scale, int32_t causal, int64_t window, void* o,
                                  int64_t ld_o, void* workspace, size_t workspace_bytes,
                                  void* stream) {
    const float score = scale * kLog2e;
    if (causal < 0 || causal > 1 || window < 0 || !(score > 0.0f) || !isfinite(score))
        return README_ERR_ARG;
    KvAttnArgs a{};
    bool done;
    const readme_status st =
        attention_args(kt, T, R, H, Hk, D, q, ld_q, offsets, lens, table, max_blocks, n_blocks, codes,
                       scales, score, window, o, ld_o, false, workspace, workspace_bytes, &a, &done);
    if (st != README_OK || done) return st;
    a.causal = causal;
    return st_of(launch_kv_attention(kt, a, as_stream(stream)));
}

size_t readme_attention_kv_tree_workspace_bytes(int64_t T, int32_t R, int32_t H, int32_t Hk,
                                                int32_t D, int64_t max_blocks) {
    bool done;
    if (kv_check_attention(README_KV_I8, T, R, H, Hk, D, max_blocks, 1, &done) != README_OK || done)
        return 0;
    return kv_attention_workspace(true, T, R, H, Hk, D, max_blocks);
}

readme_status readme_attention_kv_tree(readme_kv_type kt, int64_t T, int32_t R, int32_t H,
                                       int32_t Hk, int32_t D, const void* q, int64_t ld_q,
                                       const int32_t* offsets, const int32_t* lens,
                                       const int32_t* table, int64_t max_blocks, int64_t n_blocks,
                                       const void* codes, const float* scales,
                                       const uint64_t* tree, int32_t words, const int32_t* pos,
                                       float scale, int64_t window, void* o, int64_t ld_o,
                                       void* workspace, size_t workspace_bytes, void* stream) {
    const float score = scale * kLog2e;
    if (window < 0 || !(score > 0.0f) || !isfinite(score)) return README_ERR_ARG;
    if (words < 1) return README_ERR_ARG;
    if (words > kMaxWords) return README_ERR_UNSUPPORTED;
    KvAttnArgs a{};
    bool done;
    const readme_status st =
        attention_args(kt, T, R, H, Hk, D, q, ld_q, offsets, lens, table, max_blocks, n_blocks, codes,
                       scales, score, window, o, ld_o, true, workspace, workspace_bytes, &a, &done);
    if (st != README_OK || done) return st;
    if (!tree || !al(tree, 8) || !al(pos, 4)) return README_ERR_ARG;
    a.tree = tree;
    a.words = words;
    a.pos = pos;
    return st_of(launch_kv_attention(kt, a, as_stream(stream)));
}

}  // extern "C"
