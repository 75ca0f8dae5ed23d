// readme_verify_drafts: drafted tokens against the target's distributions.
//
// One workgroup a request.  What decides whether a draft is taken are a few numbers
// a row (t and q at its token, u), which the threads gather once, all rows together;
// the first wave then walks down the tree.  Only a refused draft asks for the whole
// distributions, to know what is left of the target's (W), and the end for the place
// of the next token.  t is not stored: refusals at one node change it by
// t = max(t - a q, 0) with an `a` each, so it is computed again from p and q wherever
// it is read.
#include <limits.h>

#include "common.hpp"
#include "internal.hpp"

using namespace readme;

namespace readme {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxRows = README_MAX_DRAFT_ROWS;

struct VerifyArgs {
    int64_t T, R, V;
    const int32_t *offsets, *tokens, *parent;
    const void *p, *q;
    int64_t ld_p, ld_q;
    const float* u;
    int distinct;
    int32_t *path, *accepted, *token;
};

__device__ __forceinline__ double positive(float x) { return x > 0.0f ? (double)x : 0.0; }

template <int DT>
__device__ __forceinline__ double entry(const void* base, int64_t at) {
    if constexpr (DT == README_F32) return positive(reinterpret_cast<const float*>(base)[at]);
    return positive(__uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(base)[at] << 16));
}

// A request's rows, and the refusals at the node that the walk stands at.
struct VerifyLds {
    int parent[kMaxRows], token[kMaxRows];
    double t[kMaxRows], q[kMaxRows];   // of the draft's token at its parent
    float u[kMaxRows];
    double a[kMaxRows];                // of each refusal
    int refused[kMaxRows];
    double sums[2][kWaves], shares[kWaves];
    int child, taken;
};

// t and q of the node at vocabulary entry v after `k` refusals.
template <int DT, bool CERTAIN>
__device__ __forceinline__ double residual(const VerifyLds& l, double p, double q, int64_t v, int k) {
    for (int j = 0; j < k; ++j) {
        if constexpr (CERTAIN) {
            if (l.refused[j] == v) p = 0.0;
        } else {
            p = fmax(p - l.a[j] * q, 0.0);
        }
    }
    return p;
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off, 64);
    return x;
}

template <int DT, bool CERTAIN>
__global__ __launch_bounds__(kThreads) void k_verify(VerifyArgs a) {
    __shared__ VerifyLds l;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int64_t r = blockIdx.x;
    int64_t lo = a.offsets[r], hi = a.offsets[r + 1];
    lo = lo < 0 ? 0 : (lo > a.T ? a.T : lo);
    hi = hi < lo ? lo : (hi > a.T ? a.T : hi);
    if (lo == hi) {
        if (tid == 0) {
            a.accepted[r] = 0;
            a.token[r] = -1;
        }
        return;
    }
    const int n = (int)(hi - lo < kMaxRows ? hi - lo : kMaxRows);
    for (int64_t i = tid; i < hi - lo; i += kThreads) a.path[lo + i] = i == 0 ? 0 : -1;
    if (tid < n) {
        const int par = a.parent[lo + tid], x = a.tokens[lo + tid];
        const bool real = tid > 0 && par >= 0 && par < tid, known = real && x >= 0 && x < a.V;
        l.parent[tid] = real ? par : -1;
        l.token[tid] = known ? x : -1;
        l.u[tid] = a.u[lo + tid];
        l.t[tid] = known ? entry<DT>(a.p, (lo + par) * a.ld_p + x) : 0.0;
        l.q[tid] = !known ? 0.0 : CERTAIN ? 1.0 : entry<DT>(a.q, (lo + par) * a.ld_q + x);
    }
    __syncthreads();
    // Each wave's part of the vocabulary, in whole steps of the waves
    const int64_t part = (a.V + kThreads - 1) / kThreads * 64;
    const int64_t v0 = wv * part < a.V ? wv * part : a.V, v1 = v0 + part < a.V ? v0 + part : a.V;

    int node = 0, last = 0, k = 0, depth = 0;
    double rate = 1.0;
    bool summed = false;  // l.sums[0] holds the waves' sums of t
    for (;;) {
        // The next draft below the node, and whether it is taken
        if (wv == 0) {
            int child = -1;
            for (int g = last / 64; g * 64 < n && child < 0; ++g) {
                const int i = g * 64 + lane;
                const uint64_t hit = __ballot(i < n && i > last && l.parent[i] == node);
                if (hit) child = g * 64 + __ffsll((unsigned long long)hit) - 1;
            }
            if (lane == 0) {
                l.child = child;
                l.taken = child >= 0 && (double)l.u[child] * rate * l.q[child] < l.t[child];
            }
        }
        __syncthreads();
        const int child = l.child;
        const bool taken = l.taken != 0;
        if (child < 0) break;
        last = child;
        if (taken) {
            ++depth;
            if (tid == 0) a.path[lo + depth] = child;
            node = child;
            k = 0;
            rate = 1.0;
            summed = false;
            __syncthreads();
            continue;
        }
        // Refused: what is left of the target's distribution, and of the drafts'
        const int x = l.token[child];
        if (tid == 0) {
            l.a[k] = rate;
            l.refused[k] = x;
        }
        __syncthreads();
        double w = 0.0, s = 0.0;
        for (int64_t v = v0 + lane; v < v1; v += 64) {
            const double p = entry<DT>(a.p, (lo + node) * a.ld_p + v);
            const double q = CERTAIN ? 0.0 : entry<DT>(a.q, (lo + node) * a.ld_q + v);
            w += residual<DT, CERTAIN>(l, p, q, v, k + 1);
            if (!CERTAIN && a.distinct) {
                bool gone = false;
                for (int j = 0; j <= k; ++j) gone = gone || l.refused[j] == v;
                s += gone ? 0.0 : q;
            }
        }
        w = wave_sum(w);
        s = wave_sum(s);
        // Not over the sums of an earlier refusal, which stay if nothing is left
        double* const sums = l.sums[(k + 1) & 1];
        double* const shares = l.shares;
        if (lane == 0) {
            sums[wv] = w;
            shares[wv] = s;
        }
        __syncthreads();
        w = s = 0.0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            w += sums[i];
            s += shares[i];
        }
        if (!(w > 0.0)) break;
        if (tid < n && l.parent[tid] == node) {
            double t = l.t[tid];
            if constexpr (CERTAIN) {
                if (l.token[tid] == x) t = 0.0;
            } else {
                t = fmax(t - rate * l.q[tid], 0.0);
                if (a.distinct && l.token[tid] == x) l.q[tid] = 0.0;
            }
            l.t[tid] = t;
        }
        rate = !CERTAIN && a.distinct ? (s > 0.0 ? w / s : 0.0) : w;
        ++k;
        summed = true;
        __syncthreads();
    }

    __syncthreads();  // the walk's last reads of l.child and l.shares are over
    // The next token: the waves' sums of t, the wave whose part holds the border,
    // the thread whose piece of that part does, and the entry.
    double* const sums = l.sums[k & 1];
    if (!summed) {
        double w = 0.0;
        for (int64_t v = v0 + lane; v < v1; v += 64) w += entry<DT>(a.p, (lo + node) * a.ld_p + v);
        w = wave_sum(w);
        __syncthreads();
        if (lane == 0) sums[wv] = w;
        __syncthreads();
    }
    double total = 0.0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) total += sums[i];
    const double border = (double)l.u[0] * total;
    double before = 0.0, run = 0.0;
    int at = -1;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        // Past the border; or, where rounding leaves none, the last that is not empty
        if (sums[i] > 0.0 && (at < 0 || !(before + sums[at] > border))) {
            at = i;
            before = run;
        }
        run += sums[i];
    }
    if (at < 0) {
        if (tid == 0) a.token[r] = -1;
    }
    if (tid == 0) a.accepted[r] = depth;
    if (at < 0) return;
    const int64_t p0 = at * part, p1 = p0 + part < a.V ? p0 + part : a.V;
    const int64_t piece = (p1 - p0 + kThreads - 1) / kThreads;
    int64_t b0 = p0 + tid * piece, b1 = b0 + piece;
    b0 = b0 < p1 ? b0 : p1;
    b1 = b1 < p1 ? b1 : p1;
    double mine = 0.0;
    for (int64_t v = b0; v < b1; ++v)
        mine += residual<DT, CERTAIN>(l, entry<DT>(a.p, (lo + node) * a.ld_p + v),
                                      CERTAIN ? 0.0 : entry<DT>(a.q, (lo + node) * a.ld_q + v), v, k);
    double incl = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const double y = __shfl_up(incl, off, 64);
        if (lane >= off) incl += y;
    }
    if (tid == 0) l.child = INT_MAX, l.taken = -1;
    if (lane == 63) l.shares[wv] = incl;
    __syncthreads();
    double from = before;
    for (int i = 0; i < wv; ++i) from += l.shares[i];
    if (mine > 0.0) {
        if (from + incl > border) atomicMin(&l.child, tid);
        atomicMax(&l.taken, tid);
    }
    __syncthreads();
    if (tid != (l.child != INT_MAX ? l.child : l.taken)) return;
    double sum = from + incl - mine;
    int64_t found = -1;
    for (int64_t v = b0; v < b1; ++v) {
        const double t = residual<DT, CERTAIN>(l, entry<DT>(a.p, (lo + node) * a.ld_p + v),
                                               CERTAIN ? 0.0 : entry<DT>(a.q, (lo + node) * a.ld_q + v), v, k);
        sum += t;
        if (t > 0.0) {
            found = v;
            if (sum > border) break;
        }
    }
    a.token[r] = (int)found;
}

inline readme_status st_of(hipError_t e) { return e == hipSuccess ? README_OK : README_ERR_HIP; }
inline bool al(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

bool sizes_ok(int64_t T, int32_t R, int64_t V) {
    return T <= (1ll << 27) && R <= (1 << 20) && V <= INT_MAX && R <= (1ll << 36) / V;
}

}  // namespace

}  // namespace readme

extern "C" {

size_t readme_verify_drafts_workspace_bytes(int64_t T, int32_t R, int64_t V) {
    if (T < 0 || R < 1 || V < 1 || !sizes_ok(T, R, V)) return 0;
    return 0;
}

readme_status readme_verify_drafts(readme_dtype dt, int64_t T, int32_t R, int64_t V,
                                   const int32_t* offsets, const int32_t* tokens,
                                   const int32_t* parent, const void* p, int64_t ld_p,
                                   const void* q, int64_t ld_q, const float* u, int32_t distinct,
                                   int32_t* path, int32_t* accepted, int32_t* token,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    if (dt != README_F32 && dt != README_BF16) return README_ERR_UNSUPPORTED;
    if (T < 0 || R < 0 || V < 1 || distinct < 0 || distinct > 1) return README_ERR_ARG;
    if (!sizes_ok(T, R, V)) return README_ERR_UNSUPPORTED;
    if (R == 0) return T == 0 ? README_OK : README_ERR_ARG;
    if (!offsets || !accepted || !token) return README_ERR_ARG;
    if (!al(offsets, 4) || !al(accepted, 4) || !al(token, 4)) return README_ERR_ARG;
    if (T > 0) {
        const int64_t es = (int64_t)dtype_size(dt);
        if (!tokens || !parent || !p || !u || !path) return README_ERR_ARG;
        if (!al(tokens, 4) || !al(parent, 4) || !al(u, 4) || !al(path, 4)) return README_ERR_ARG;
        if (!al(p, 16) || !al(q, 16)) return README_ERR_ARG;
        if (ld_p < V || ld_p * es % 16 != 0) return README_ERR_ARG;
        if (q && (ld_q < V || ld_q * es % 16 != 0)) return README_ERR_ARG;
    }
    if (!al(workspace, 16)) return README_ERR_ARG;
    const size_t need = readme_verify_drafts_workspace_bytes(T, R, V);
    if (need > 0 && !workspace) return README_ERR_ARG;
    if (workspace_bytes < need) return README_ERR_WORKSPACE;
    VerifyArgs a;
    a.T = T;
    a.R = R;
    a.V = V;
    a.offsets = offsets;
    a.tokens = tokens;
    a.parent = parent;
    a.p = p;
    a.q = q;
    a.ld_p = ld_p;
    a.ld_q = ld_q;
    a.u = u;
    a.distinct = distinct;
    a.path = path;
    a.accepted = accepted;
    a.token = token;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (dt == README_F32) {
        if (q) k_verify<README_F32, false><<<(unsigned)R, kThreads, 0, s>>>(a);
        else k_verify<README_F32, true><<<(unsigned)R, kThreads, 0, s>>>(a);
    } else {
        if (q) k_verify<README_BF16, false><<<(unsigned)R, kThreads, 0, s>>>(a);
        else k_verify<README_BF16, true><<<(unsigned)R, kThreads, 0, s>>>(a);
    }
    return st_of(hipGetLastError());
}

}  // extern "C"
