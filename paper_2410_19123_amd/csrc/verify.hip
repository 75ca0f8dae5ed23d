// readme_verify_drafts: drafted tokens against the target's distributions.
//
// One workgroup a request.  What decides whether a draft is taken are a few numbers
// a row (t and q at its token, u), which the threads gather once, all rows together;
// the first wave then walks down the tree by itself until a draft is refused or none
// is left.  Only a refused draft asks for the whole distributions, to know what is
// left of the target's (W), and the end for the place of the next token.  t is not
// stored: as q >= 0, the refusals at a node, t = max(t - a q, 0) with an `a` each,
// come to t = max(p - A q, 0) with A the sum of their a, so it is computed from p and
// q wherever it is read.
// A workgroup's waves hold a part of the vocabulary each; a pass leaves the parts'
// sums, from which the end knows the part that holds the next token.  What loses one
// token by a refusal, the sum of q without the refused or, of certain drafts, t
// itself, is summed anew in the part that held it alone.
//
// A request's refusals wait for each other, each factor for the sum before it, so a
// request has one CU and its vector ALU is the bound: a refusal over 100003 entries in
// bf16 costs 8 us, ten instructions an entry (both unpacked, converted to fp64, q held
// at 0, the product, the maximum, the sum), over 32000 3.5; of a certain draft 2.5, which
// sums one part anew.  64 chains of 5 drafts over 32000 fp32 entries 12.4, 16 MB; 24
// trees of 17 to 33 rows over 100003 40 to 60, the request that is refused most, where
// the requests' mean is about half of that.  Steps on the way, these two: entry by entry
// 30 and 226, 16-byte loads and the first wave's walk 16 and 75.
// A request over several CUs would need them to wait for one another at every refusal,
// in a launch that does not promise that all of them run.  Not tried: a list of the
// entries that are left for a node's later refusals.  In the trees above 64% are left
// after a node's first refusal, 50% after its second, 41% after its third, and 31 of 44
// refusals are their node's first, which such a list does not shorten.
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

// Consecutive entries of a row, 16 bytes of them, as they are stored; fewer, and zeros,
// at the row's end, past which nothing is read.
template <int DT>
constexpr int kRun = DT == README_F32 ? 4 : 8;
template <int DT>
__device__ __forceinline__ uint4 load_run(const void* row, int64_t v) {
    return *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(row) + v * (16 / kRun<DT>));
}
template <int DT>
__device__ __forceinline__ uint4 load_tail(const void* row, int64_t v, int n) {
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < kRun<DT>; ++e) {
        if (e >= n) break;
        if constexpr (DT == README_F32)
            w[e] = reinterpret_cast<const uint32_t*>(row)[v + e];
        else
            w[e >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[v + e] << (16 * (e & 1));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <int DT>
__device__ __forceinline__ double run_raw(const uint4& r, int e) {
    const int d = DT == README_F32 ? e : e >> 1;
    const uint32_t w = d == 0 ? r.x : d == 1 ? r.y : d == 2 ? r.z : r.w;
    return (double)(DT == README_F32 ? __uint_as_float(w) : e & 1 ? bf16_hi(w) : bf16_lo(w));
}
template <int DT>
__device__ __forceinline__ double run_at(const uint4& r, int e) {
    return fmax(run_raw<DT>(r, e), 0.0);  // a NaN gives 0
}

// A request's rows, and the refusals at the node that the walk stands at.
struct VerifyLds {
    int parent[kMaxRows], token[kMaxRows];
    double p[kMaxRows], q[kMaxRows];   // of the draft's token at its parent
    float u[kMaxRows];
    int refused[kMaxRows];
    double sums[2][kWaves], shares[kWaves], again[kWaves];
    int node, child, depth;            // where the walk stands, the draft refused or -1
    int found;
};

// 0 for p below 0 or NaN too.
__device__ __forceinline__ double left_over(double p, double q, double A) { return fmax(fma(-A, q, p), 0.0); }

// The run x at v without the first k refused tokens.
template <int DT>
__device__ __forceinline__ void without(const VerifyLds& l, const uint4& x, int64_t v, int k,
                                        double (&y)[kRun<DT>]) {
    constexpr int E = kRun<DT>;
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = run_at<DT>(x, e);
    for (int j = 0; j < k; ++j) {
        const int64_t at = (int64_t)l.refused[j] - v;
        if (!__any(at >= 0 && at < E)) continue;  // for most runs of most waves
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = at == e ? 0.0 : y[e];
    }
}
// t of the run at v after k refusals at its node, the sum of whose a is A.
template <int DT, bool CERTAIN>
__device__ __forceinline__ void residual(const VerifyLds& l, const uint4& p, const uint4& q, int64_t v,
                                         int k, double A, double (&t)[kRun<DT>]) {
    if constexpr (CERTAIN) {
        without<DT>(l, p, v, k, t);
    } else {
#pragma unroll
        for (int e = 0; e < kRun<DT>; ++e) t[e] = left_over(run_raw<DT>(p, e), run_at<DT>(q, e), A);
    }
}

// Lane i the sum over lanes 0 .. i, by the lanes' own network: within rows of 16, then
// from row to row.
template <int CTRL, int ROWS>
__device__ __forceinline__ double add_from(double x) {
    const int64_t b = __double_as_longlong(x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, ROWS, 0xf, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xf, true);
    return x + __longlong_as_double((int64_t)(((uint64_t)hi << 32) | lo));
}
__device__ __forceinline__ double wave_scan(double x) {
    x = add_from<0x111, 0xf>(x);  // row_shr:1
    x = add_from<0x112, 0xf>(x);
    x = add_from<0x114, 0xf>(x);
    x = add_from<0x118, 0xf>(x);
    x = add_from<0x142, 0xa>(x);  // row_bcast:15 into rows 1 and 3
    return add_from<0x143, 0xc>(x);  // row_bcast:31 into rows 2 and 3
}
__device__ __forceinline__ double sum_of(const double (&x)[kWaves]) {
    double s[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
    for (int i = 4; i < kWaves; ++i) s[i & 3] += x[i];
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// Calls f(v, p, q) for the lane's runs of the entries v0 .. v0 + len - 1 (one of the
// parts, so len fits 32 bits): in steps of 64 runs at `first`, first + stride, ..; the
// next kBatch steps are on their way meanwhile.
constexpr int kBatch = 2;
template <int DT, bool CERTAIN, class F>
__device__ __forceinline__ void for_runs(const void* p, const void* q, int64_t v0, int len, int first,
                                         int stride, F&& f) {
    constexpr int E = kRun<DT>, B = kBatch;
    const int full = len / E * E;
    p = reinterpret_cast<const char*>(p) + v0 * (16 / E);
    if constexpr (!CERTAIN) q = reinterpret_cast<const char*>(q) + v0 * (16 / E);
    struct Batch {
        uint4 p[B], q[B];
    } a, b;
    const int mine = (threadIdx.x & 63) * E;
    // Past the last whole run the loads repeat it
    auto fetch = [&](int at, Batch& x) {
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int v = min(at + i * stride + mine, full - E);
            const uint32_t byte = (uint32_t)v * (16 / E);
            x.p[i] = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(p) + byte);
            if constexpr (!CERTAIN) x.q[i] = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(q) + byte);
        }
    };
    auto use = [&](int at, const Batch& x) {
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int v = at + i * stride + mine;
            if (v < full) f(v0 + v, x.p[i], CERTAIN ? x.p[i] : x.q[i]);
        }
    };
    if (first < full) {
        fetch(first, a);
        for (int at = first;;) {
            const int after = at + B * stride;
            if (after >= full) {
                use(at, a);
                break;
            }
            fetch(after, b);
            use(at, a);
            at = after + B * stride;
            if (at >= full) {
                use(after, b);
                break;
            }
            fetch(at, a);
            use(after, b);
        }
    }
    // What is left of the row, by the first lane whose step it would be
    if (full < len && (full / (64 * E)) % (stride / (64 * E)) == first / (64 * E) && mine == full % (64 * E)) {
        const uint4 tp = load_tail<DT>(p, full, len - full);
        f(v0 + full, tp, CERTAIN ? tp : load_tail<DT>(q, full, len - full));
    }
}

template <int DT, bool CERTAIN>
__global__ __launch_bounds__(kThreads) void k_verify(VerifyArgs a) {
    constexpr int E = kRun<DT>;
    __shared__ VerifyLds l;
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
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
        l.p[tid] = known ? entry<DT>(a.p, (lo + par) * a.ld_p + x) : 0.0;
        l.q[tid] = !known ? 0.0 : CERTAIN ? 1.0 : entry<DT>(a.q, (lo + par) * a.ld_q + x);
    }
    __syncthreads();
    // Each wave's part of the vocabulary, in whole steps of its lanes' runs
    constexpr int kStep = 64 * E;
    const int64_t part = (a.V + kWaves * kStep - 1) / (kWaves * kStep) * kStep;  // at most 2^27 + kStep
    const int64_t v0 = wv * part < a.V ? wv * part : a.V;
    auto length = [&](int64_t from) { return (int)(a.V - from < part ? a.V - from : part); };
    const int len = length(v0);
    constexpr int es = 16 / E;
    auto row_of = [&](const void* base, int64_t ld, int node) {
        return reinterpret_cast<const void*>(reinterpret_cast<const char*>(base) + (lo + node) * ld * es);
    };

    int node = 0, last = 0, k = 0, depth = 0;
    double rate = 1.0, A = 0.0;  // a, and the sum of the refusals'
    const bool loses = CERTAIN || a.distinct;  // p or q loses the refused token
    int pending = -1;                          // the part whose sum is `changed`
    double changed = 0.0;
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
                if (child < 0) break;
                double t = CERTAIN ? l.p[child] : left_over(l.p[child], l.q[child], A), qx = l.q[child];
                if (loses) {  // a token refused before has lost its p, or q
                    bool gone = false;
                    for (int j = lane; j - lane < k; j += 64)
                        gone = gone || __ballot(j < k && l.refused[j] == l.token[child]) != 0;
                    if (gone) t = qx = 0.0;
                }
                if (!((double)l.u[child] * rate * qx < t)) break;
                ++depth;
                if (lane == 0) a.path[lo + depth] = child;
                node = last = child;
                k = 0;
                rate = 1.0;
                A = 0.0;
                pending = -1;
            }
            if (lane == 0) {
                l.node = node;
                l.child = child;
                l.depth = depth;
                if (child >= 0) l.refused[k] = l.token[child];  // the refusal that comes next
            }
        }
        __syncthreads();
        if (l.depth != depth) k = 0, rate = 1.0, A = 0.0, pending = -1;
        // The part that the last refusal changed, now that its old sum is read no more
        if (!CERTAIN && pending >= 0 && tid == 0) l.shares[pending] = changed;
        // The same for all lanes, and so are the rows' addresses
        node = __builtin_amdgcn_readfirstlane(l.node);
        depth = __builtin_amdgcn_readfirstlane(l.depth);
        const int child = __builtin_amdgcn_readfirstlane(l.child);
        if (child < 0) break;
        last = child;
        // Refused: what is left of the target's distribution, and of the drafts'
        const void *p = row_of(a.p, a.ld_p, node), *q = CERTAIN ? nullptr : row_of(a.q, a.ld_q, node);
        const int x = __builtin_amdgcn_readfirstlane(l.token[child]);
        const double A1 = A + rate;
        if (!CERTAIN || k == 0) {
            const bool first = !CERTAIN && a.distinct && k == 0;
            double w = 0.0, s = 0.0;
            for_runs<DT, CERTAIN>(p, q, v0, len, 0, kStep, [&](int64_t v, const uint4& rp, const uint4& rq) {
                double t[E];
                residual<DT, CERTAIN>(l, rp, rq, v, k + 1, A1, t);
#pragma unroll
                for (int e = 0; e < E; ++e) w += t[e];
                if (first) {
                    without<DT>(l, rq, v, k + 1, t);
#pragma unroll
                    for (int e = 0; e < E; ++e) s += t[e];
                }
            });
            w = wave_scan(w);
            if (lane == 63) l.sums[(k + 1) & 1][wv] = w;
            if (first) {
                s = wave_scan(s);
                if (lane == 63) l.shares[wv] = s;
            }
        } else if (lane == 63) {
            l.sums[(k + 1) & 1][wv] = wv == pending ? changed : l.sums[k & 1][wv];
        }
        // Of the others only the part that held x changes: summed anew by all waves
        const int at = loses && k > 0 && x >= 0 ? (int)(x / part) : -1;
        if (at >= 0) {
            double s = 0.0;
            for_runs<DT, true>(CERTAIN ? p : q, nullptr, at * part, length(at * part), wv * kStep, kWaves * kStep,
                               [&](int64_t v, const uint4& run, const uint4&) {
                                   double y[E];
                                   without<DT>(l, run, v, k + 1, y);
#pragma unroll
                                   for (int e = 0; e < E; ++e) s += y[e];
                               });
            s = wave_scan(s);
            if (lane == 63) l.again[wv] = s;
        }
        __syncthreads();
        // From here to the barrier after the next walk only these sums are read
        double part_sums[2][kWaves];
        const double now = at >= 0 ? sum_of(l.again) : 0.0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            part_sums[0][i] = CERTAIN && i == at ? now : l.sums[(k + 1) & 1][i];
            part_sums[1][i] = !CERTAIN && i == at ? now : l.shares[i];
        }
        const double w = sum_of(part_sums[0]);
        if (!(w > 0.0)) break;
        const double s = sum_of(part_sums[1]);
        A = A1;
        rate = !CERTAIN && a.distinct ? (s > 0.0 ? w / s : 0.0) : w;
        ++k;
        pending = at;
        changed = now;
    }
    __syncthreads();  // the walk's last reads of l are over
    if (pending >= 0 && CERTAIN && tid == 0) l.sums[k & 1][pending] = changed;

    // The next token: the parts' sums of t, the part that holds the border, and in it
    // the step, the lane and the entry.
    const void *p = row_of(a.p, a.ld_p, node), *q = CERTAIN ? nullptr : row_of(a.q, a.ld_q, node);
    double(&sums)[kWaves] = l.sums[k & 1];
    if (k == 0) {
        double w = 0.0;
        for_runs<DT, true>(p, nullptr, v0, len, 0, kStep, [&](int64_t, const uint4& rp, const uint4&) {
#pragma unroll
            for (int e = 0; e < E; ++e) w += run_at<DT>(rp, e);
        });
        w = wave_scan(w);
        if (lane == 63) sums[wv] = w;
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
            auto run = [&](const void* row) {
                return v + E <= p1 ? load_run<DT>(row, v) : load_tail<DT>(row, v, (int)(p1 - v));
            };
            const uint4 rp = run(p);
            const uint4 rq = CERTAIN || k == 0 ? make_uint4(0u, 0u, 0u, 0u) : run(q);
            residual<DT, CERTAIN>(l, rp, rq, v, k, A, t);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) mine += t[e];
        const double incl = wave_scan(mine);
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

// A request's state is in its workgroup's LDS.
size_t readme_verify_drafts_workspace_bytes(int64_t, int32_t, int64_t) { return 0; }

readme_status readme_verify_drafts(readme_dtype dt, int64_t T, int32_t R, int64_t V,
                                   const int32_t* offsets, const int32_t* tokens,
                                   const int32_t* parent, const void* p, int64_t ld_p,
                                   const void* q, int64_t ld_q, const float* u, int32_t distinct,
                                   int32_t* path, int32_t* accepted, int32_t* token,
                                   void* workspace, size_t, void* stream) {
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
