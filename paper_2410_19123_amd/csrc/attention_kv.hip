// Attention over the 8-bit cache: which kernel a call takes, its workspace, and
// the join of partial results.
#include <math.h>

#include "attention_kv.hpp"

namespace readme {

namespace {

// Joins the parts of each pair that several workgroups shared, and zeroes the
// rows of a request that sees no block.  One workgroup per (row tile slot,
// head); thread i takes four dims of one row at a time.
template <int D, int ROWS>
__global__ __launch_bounds__(256) void k_attention_join(KvAttnArgs a, const int64_t* __restrict__ plan,
                                                        const float* __restrict__ parts) {
    constexpr int kPart = kv_part_floats<D, ROWS>;
    const int h = blockIdx.y;
    int64_t tl;
    const int64_t r = kv_slot_request<ROWS>(a, blockIdx.x, tl);
    const KvRequest q = kv_request(a, r);
    const KvPlan p = kv_plan<ROWS>(a, q);
    if (tl < 0 || tl >= p.tiles) return;
    int64_t g0 = 0, g1 = -1;
    if (p.blocks > 0) {
        const int64_t share = plan[0];
        const int64_t s = plan[1 + r] + (tl * a.c.Hk + h) * p.blocks;
        g0 = s / share;
        g1 = (s + p.blocks - 1) / share;
        if (g0 == g1) return;
    }
    // Part of workgroup g: its second where the pair begins in its share.
    auto part = [&](int64_t g) { return parts + (g * 2 + (g == g0 ? 1 : 0)) * kPart; };
    const int rows = (int)((int64_t)q.n * a.G - tl * ROWS < ROWS ? (int64_t)q.n * a.G - tl * ROWS : ROWS);
    for (int e = threadIdx.x; e < rows * (D / 4); e += 256) {
        const int i = e / (D / 4), d = e % (D / 4) * 4;
        float m = -INFINITY;
        for (int64_t g = g0; g <= g1; ++g) m = fmaxf(m, part(g)[ROWS * D + i]);
        const float base = m == -INFINITY ? 0.0f : m;
        float l = 0.0f;
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int64_t g = g0; g <= g1; ++g) {
            const float* pp = part(g);
            const float f = __builtin_amdgcn_exp2f(pp[ROWS * D + i] - base);
            l = fmaf(pp[ROWS * (D + 1) + i], f, l);
            acc += *reinterpret_cast<const f32x4*>(pp + i * D + d) * f;
        }
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        const int64_t row = tl * ROWS + i;
        const int64_t tok = row / a.G, head = (int64_t)h * a.G + row - tok * a.G;
        uint2 w;
        w.x = (uint32_t)f32_to_bf16(acc[0] * inv) | ((uint32_t)f32_to_bf16(acc[1] * inv) << 16);
        w.y = (uint32_t)f32_to_bf16(acc[2] * inv) | ((uint32_t)f32_to_bf16(acc[3] * inv) << 16);
        *reinterpret_cast<uint2*>(a.o + (q.row0 + tok) * a.ld_o + head * D + d) = w;
    }
}

template <int D>
hipError_t join_of(const KvAttnArgs& a, int rows, hipStream_t s) {
    const int64_t* plan = reinterpret_cast<const int64_t*>(a.ws);
    const float* parts =
        reinterpret_cast<const float*>(reinterpret_cast<const char*>(a.ws) + kv_plan_bytes(a.c.R));
    const dim3 grid((unsigned)kv_slots(a.c.T, a.c.R, a.G, rows), (unsigned)a.c.Hk);
    if (rows == kRowsTile) k_attention_join<D, kRowsTile><<<grid, 256, 0, s>>>(a, plan, parts);
    else k_attention_join<D, kTilesTile><<<grid, 256, 0, s>>>(a, plan, parts);
    return hipGetLastError();
}

hipError_t launch_join(const KvAttnArgs& a, int rows, hipStream_t s) {
    switch (a.c.D) {
        case 64: return join_of<64>(a, rows, s);
        case 128: return join_of<128>(a, rows, s);
        case 256: return join_of<256>(a, rows, s);
    }
    return hipErrorInvalidValue;
}

// What a call runs, from the sizes the host knows.
enum Form { FORM_ROWS, FORM_TILES_SHARES, FORM_TILES_WHOLE };

Form form_of(int64_t T, int64_t R, int64_t G, int64_t Hk) {
    if (T * G <= R * kRowsTile) return FORM_ROWS;
    if (kv_slots(T, R, G, kTilesTile) * Hk >= 2 * kTilesShares) return FORM_TILES_WHOLE;
    return FORM_TILES_SHARES;
}

}  // namespace

size_t kv_attention_workspace(int64_t T, int64_t R, int H, int Hk, int D, int64_t max_blocks) {
    (void)max_blocks;
    const Form f = form_of(T, R, H / Hk, Hk);
    const int64_t rows = f == FORM_ROWS           ? kRowsShares * kRowsTile
                         : f == FORM_TILES_SHARES ? kTilesShares * kTilesTile
                                                  : 0;
    return (size_t)(kv_plan_bytes(R) + 2 * rows * (D + 2) * 4);
}

hipError_t launch_kv_attention(readme_kv_type kt, const KvAttnArgs& a, hipStream_t s) {
    const Form f = form_of(a.c.T, a.c.R, a.G, a.c.Hk);
    if (f == FORM_TILES_WHOLE) return launch_attention_tiles(kt, a, false, s);
    const hipError_t e = f == FORM_ROWS ? launch_attention_rows(kt, a, s)
                                          : launch_attention_tiles(kt, a, true, s);
    return e != hipSuccess ? e : launch_join(a, f == FORM_ROWS ? kRowsTile : kTilesTile, s);
}

}  // namespace readme
