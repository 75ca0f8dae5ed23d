// readme_verify_drafts: drafted tokens against the target's distributions.
//
// One workgroup a request.  What decides whether a draft is taken are a few numbers
// a row (t and q at its token, u), which the threads gather once, all rows together;
// the first wave then walks down the tree by itself until a draft is refused or none
// is left.  Only a refused draft asks for the whole distributions, to know what is
// left of the target's (W), and the end for the place of the next token.  t is not
// stored: refusals at one node change it by t = max(t - a q, 0) with an `a` each, so
// it is computed again from p and q wherever it is read.
// A workgroup's waves hold a part of the vocabulary each; a pass leaves the parts'
// sums, from which the end knows the part that holds the next token.
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

// Consecutive entries of a row, 16 bytes of them, as they are stored.
template <int DT>
constexpr int kRun = DT == README_F32 ? 4 : 8;
template <int DT>
__device__ __forceinline__ uint4 load_run(const void* row, int64_t v, int64_t end) {
    const char* at = reinterpret_cast<const char*>(row) + v * (16 / kRun<DT>);
    if (v + kRun<DT> <= end) return *reinterpret_cast<const uint4*>(at);
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < kRun<DT>; ++e) {
        if (v + e >= end) break;
        if constexpr (DT == README_F32)
            w[e] = reinterpret_cast<const uint32_t*>(at)[e];
        else
            w[e >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(at)[e] << (16 * (e & 1));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <int DT>
__device__ __forceinline__ double run_at(const uint4& r, int e) {
    const int d = DT == README_F32 ? e : e >> 1;
    const uint32_t w = d == 0 ? r.x : d == 1 ? r.y : d == 2 ? r.z : r.w;
    const float x = DT == README_F32 ? __uint_as_float(w) : e & 1 ? bf16_hi(w) : bf16_lo(w);
    return (double)fmaxf(x, 0.0f);  // a NaN gives 0
}

// A request's rows, and the refusals at the node that the walk stands at.
struct VerifyLds {
    int parent[kMaxRows], token[kMaxRows];
    double t[kMaxRows], q[kMaxRows];   // of the draft's token at its parent
    float u[kMaxRows];
    double a[kMaxRows];                // of each refusal
    int refused[kMaxRows];
    double sums[2][kWaves], shares[kWaves];
    int node, child, depth;            // where the walk stands, the draft refused or -1
    int found;
};

// t of the run at v after `k` refusals at its node.
template <int DT, bool CERTAIN>
__device__ __forceinline__ void residual(const VerifyLds& l, const uint4& p, const uint4& q, int64_t v,
                                         int k, double (&t)[kRun<DT>]) {
    constexpr int E = kRun<DT>;
#pragma unroll
    for (int e = 0; e < E; ++e) t[e] = run_at<DT>(p, e);
    for (int j = 0; j < k; ++j) {
        if constexpr (CERTAIN) {
            const int64_t x = l.refused[j] - v;
#pragma unroll
            for (int e = 0; e < E; ++e) t[e] = x == e ? 0.0 : t[e];
        } else {
            const double a = l.a[j];
#pragma unroll
            for (int e = 0; e < E; ++e) t[e] = fmax(fma(-a, run_at<DT>(q, e), t[e]), 0.0);
        }
    }
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off, 64);
    return x;
}
__device__ __forceinline__ double sum_of(const double (&x)[kWaves]) {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) s += x[i];
    return s;
}

// Calls f(v, p, q) for the lane's runs of [v0, v1): kBatch runs of p and of q are
// on their way together.
constexpr int kBatch = 4;
template <int DT, bool CERTAIN, class F>
__device__ __forceinline__ void for_runs(const void* p, const void* q, int64_t v0, int64_t v1, F&& f) {
    constexpr int64_t kStep = 64 * kRun<DT>;
    for (int64_t v = v0 + (threadIdx.x & 63) * kRun<DT>; v < v1; v += kBatch * kStep) {
        uint4 rp[kBatch], rq[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            rp[i] = rq[i] = make_uint4(0u, 0u, 0u, 0u);
            if (v + i * kStep >= v1) continue;
            rp[i] = load_run<DT>(p, v + i * kStep, v1);
            if constexpr (!CERTAIN) rq[i] = load_run<DT>(q, v + i * kStep, v1);
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            if (v + i * kStep < v1) f(v + i * kStep, rp[i], rq[i]);
    }
}

template <int DT, bool CERTAIN>
__global__ __launch_bounds__(kThreads) void k_verify(VerifyArgs a) {
    constexpr int E = kRun<DT>;
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
    // Each wave's part of the vocabulary, in whole steps of its lanes' runs
    constexpr int64_t kStep = 64 * E;
    const int64_t part = (a.V + kWaves * kStep - 1) / (kWaves * kStep) * kStep;
    const int64_t v0 = wv * part < a.V ? wv * part : a.V, v1 = v0 + part < a.V ? v0 + part : a.V;
    constexpr int es = 16 / E;
    auto row_of = [&](const void* base, int64_t ld, int node) {
        return reinterpret_cast<const void*>(reinterpret_cast<const char*>(base) + (lo + node) * ld * es);
    };

    int node = 0, last = 0, k = 0, depth = 0;
    double rate = 1.0, all = 0.0, gone = 0.0;  // sums of q at the node, and of its refused tokens
    for (;;) {
        // The first wave: on while drafts are taken
        if (wv == 0) {
            int child;
            for (;;) {
                child = -1;
                for (int g = last / 64; g * 64 < n && child < 0; ++g) {
                    const int i = g * 64 + lane;
                    const uint64_t hit = __ballot(i < n && i > last && l.parent[i] == node);
                    if (hit) child = g * 64 + __ffsll((unsigned long long)hit) - 1;
                }
                if (child < 0 || !((double)l.u[child] * rate * l.q[child] < l.t[child])) break;
                ++depth;
                if (lane == 0) a.path[lo + depth] = child;
                node = last = child;
                k = 0;
                rate = 1.0;
            }
            if (lane == 0) {
                l.node = node;
                l.child = child;
                l.depth = depth;
                if (child >= 0) {  // the refusal that comes next
                    l.a[k] = rate;
                    l.refused[k] = l.token[child];
                }
            }
        }
        __syncthreads();
        if (l.node != node || l.depth != depth) k = 0, rate = 1.0;
        node = l.node;
        depth = l.depth;
        const int child = l.child;
        if (child < 0) break;
        last = child;
        // Refused: what is left of the target's distribution, and of the drafts'
        const void *p = row_of(a.p, a.ld_p, node), *q = CERTAIN ? nullptr : row_of(a.q, a.ld_q, node);
        const bool first = k == 0 && !CERTAIN && a.distinct;
        double w = 0.0, s = 0.0;
        for_runs<DT, CERTAIN>(p, q, v0, v1, [&](int64_t v, const uint4& rp, const uint4& rq) {
            double t[E];
            residual<DT, CERTAIN>(l, rp, rq, v, k + 1, t);
#pragma unroll
            for (int e = 0; e < E; ++e) w += t[e];
            if (first) {
#pragma unroll
                for (int e = 0; e < E; ++e) s += run_at<DT>(rq, e);
            }
        });
        w = wave_sum(w);
        if (first) s = wave_sum(s);
        // Not over the sums of an earlier refusal, which stay if nothing is left
        if (lane == 0) {
            l.sums[(k + 1) & 1][wv] = w;
            l.shares[wv] = s;
        }
        __syncthreads();
        w = sum_of(l.sums[(k + 1) & 1]);
        if (first) all = sum_of(l.shares);
        if (!(w > 0.0)) break;
        const int x = l.token[child];
        const double refused_q = l.q[child];
        __syncthreads();
        if (tid < n && l.parent[tid] == node) {
            double t = l.t[tid];
            if constexpr (CERTAIN) {
                if (l.token[tid] == x) t = 0.0;
            } else {
                t = fmax(fma(-rate, l.q[tid], t), 0.0);
                if (a.distinct && l.token[tid] == x) l.q[tid] = 0.0;
            }
            l.t[tid] = t;
        }
        rate = w;
        if (!CERTAIN && a.distinct) {
            gone = k == 0 ? refused_q : gone + refused_q;
            s = all - gone;
            if (s < all * 0x1p-10) {
                // Little is left: anew, without the cancellation
                s = 0.0;
                for_runs<DT, true>(q, nullptr, v0, v1, [&](int64_t v, const uint4& rq, const uint4&) {
                    double y[E];
                    residual<DT, true>(l, rq, rq, v, k + 1, y);
#pragma unroll
                    for (int e = 0; e < E; ++e) s += y[e];
                });
                s = wave_sum(s);
                if (lane == 0) l.shares[wv] = s;
                __syncthreads();
                s = sum_of(l.shares);
            }
            rate = s > 0.0 ? w / s : 0.0;
        }
        ++k;
        __syncthreads();
    }
    __syncthreads();  // the walk's last reads of l are over

    // The next token: the parts' sums of t, the part that holds the border, and in it
    // the step, the lane and the entry.
    const void *p = row_of(a.p, a.ld_p, node), *q = CERTAIN ? nullptr : row_of(a.q, a.ld_q, node);
    double(&sums)[kWaves] = l.sums[k & 1];
    if (k == 0) {
        double w = 0.0;
        for_runs<DT, true>(p, nullptr, v0, v1, [&](int64_t, const uint4& rp, const uint4&) {
#pragma unroll
            for (int e = 0; e < E; ++e) w += run_at<DT>(rp, e);
        });
        w = wave_sum(w);
        if (lane == 0) sums[wv] = w;
    }
    if (tid == 0) {
        l.found = -1;
        a.accepted[r] = depth;
    }
    __syncthreads();
    const double border = (double)l.u[0] * sum_of(sums);
    // The first of the waves past the border; where rounding leaves none, the last
    // that is not empty
    auto choose = [&](const double (&x)[kWaves], double& before) {
        int at = -1;
        double run = before;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            if (x[i] > 0.0 && (at < 0 || !(before + x[at] > border))) {
                at = i;
                before = run;
            }
            run += x[i];
        }
        return at;
    };
    double before = 0.0;
    const int at = choose(sums, before);
    if (at < 0) {
        if (tid == 0) a.token[r] = -1;
        return;
    }
    const int64_t p0 = at * part, p1 = p0 + part < a.V ? p0 + part : a.V;
    for (int64_t s0 = p0; s0 < p1; s0 += kWaves * kStep) {
        const int64_t v = s0 + wv * kStep + lane * E;
        double t[E], mine = 0.0;
#pragma unroll
        for (int e = 0; e < E; ++e) t[e] = 0.0;
        if (v < p1) {
            const uint4 rp = load_run<DT>(p, v, p1);
            residual<DT, CERTAIN>(l, rp, CERTAIN ? rp : load_run<DT>(q, v, p1), v, k, t);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) mine += t[e];
        double incl = mine;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const double y = __shfl_up(incl, off, 64);
            if (lane >= off) incl += y;
        }
        __syncthreads();  // an earlier step's reads of l.shares are over
        if (lane == 63) l.shares[wv] = incl;
        __syncthreads();
        double from = before;
        const int w = choose(l.shares, from);
        const bool last_step = s0 + kWaves * kStep >= p1;
        const bool here = w >= 0 && (from + l.shares[w] > border);
        if (here && wv == w) {
            // The first lane past the border, and its first entry past it
            const uint64_t past = __ballot(mine > 0.0 && from + incl > border);
            const uint64_t some = __ballot(mine > 0.0);
            const int pick = past ? __ffsll((unsigned long long)past) - 1
                                  : 63 - __clzll((long long)some);
            if (lane == pick) {
                double sum = from + incl - mine;
                int64_t found = v;
                bool done = false;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    sum += t[e];
                    if (!done && t[e] > 0.0) {
                        found = v + e;
                        done = sum > border;
                    }
                }
                a.token[r] = (int)found;
            }
        }
        if (here) return;
        // No entry past the border: the last of the part that is not 0
        int64_t most = -1;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (t[e] > 0.0) most = v + e;
        if (most >= 0) atomicMax(&l.found, (int)most);
        if (last_step) {
            __syncthreads();
            if (tid == 0) a.token[r] = l.found;
            return;
        }
        before += sum_of(l.shares);
    }
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
