// Attention over the 8-bit cache: which kernel a call takes, its workspace, and
// the join of partial results.
#include <math.h>

#include "attention_kv.hpp"

namespace readme {

namespace {

// Joins the parts of each pair that several workgroups shared, and zeroes the
// rows of a request that sees no block.  One workgroup per (tile slot, head,
// 1024 / D rows); a thread takes four dims of one row, four parts at a time in
// flight.
template <int D, int ROWS>
__global__ __launch_bounds__(256) void k_attention_join(KvAttnArgs a, const int64_t* __restrict__ plan,
                                                        const float* __restrict__ parts) {
    constexpr int kPart = kv_part_floats<D, ROWS>;
    constexpr int kStep = 1024 / D;
    const int h = blockIdx.y;
    int64_t r, tl;
    const KvRequest q = kv_slot_request<ROWS>(a, blockIdx.x, r, tl);
    const KvPlan p = kv_plan<ROWS>(a, q);
    const int i = (int)blockIdx.z * kStep + threadIdx.x / (D / 4);
    const int64_t row = tl * ROWS + i;
    if (tl < 0 || row >= (int64_t)q.n * a.G) return;
    const int d = threadIdx.x % (D / 4) * 4;
    float m = -INFINITY, l = 0.0f, unit = 0.0f;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    if (p.blocks > 0) {
        const int64_t share = plan[0];
        const int64_t s = plan[1 + r] + (tl * a.c.Hk + h) * (p.blocks + kPairCost) + kPairCost;
        const int64_t g0 = s / share, g1 = (s + p.blocks - 1) / share;
        if (g0 == g1) return;
        // Workgroup g's part is its second where the pair's first block is in
        // its share.
        for (int64_t g = g0; g <= g1; g += 4) {
            float pm[4], pl[4], pu[4];
            f32x4 pa[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t gk = g + k <= g1 ? g + k : g1;
                const float* pp = parts + (gk * 2 + (gk == g0 ? 1 : 0)) * kPart;
                pm[k] = g + k <= g1 ? pp[ROWS * D + i] : -INFINITY;
                pl[k] = pp[ROWS * (D + 1) + i];
                pu[k] = pp[ROWS * (D + 2) + i];
                pa[k] = *reinterpret_cast<const f32x4*>(pp + i * D + d);
            }
            float mn = m, un = unit;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                mn = fmaxf(mn, pm[k]);
                un = fmaxf(un, pu[k]);
            }
            const float base = mn == -INFINITY ? 0.0f : mn;
            const float f = __builtin_amdgcn_exp2f(m - base);
            m = mn;
            l *= f;
            acc *= f * unit_ratio(unit, un);
            unit = un;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float fk = __builtin_amdgcn_exp2f(pm[k] - base);
                l = fmaf(pl[k], fk, l);
                acc += pa[k] * (fk * unit_ratio(pu[k], un));
            }
        }
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int64_t tok = row / a.G, head = (int64_t)h * a.G + row - tok * a.G;
    *reinterpret_cast<uint2*>(a.o + (q.row0 + tok) * a.ld_o + head * D + d) =
        pack_bf16(acc[0] * inv * unit, acc[1] * inv * unit, acc[2] * inv * unit, acc[3] * inv * unit);
}

template <int D, int ROWS>
hipError_t join_of(const KvAttnArgs& a, hipStream_t s) {
    const int64_t* plan = reinterpret_cast<const int64_t*>(a.ws);
    const float* parts =
        reinterpret_cast<const float*>(reinterpret_cast<const char*>(a.ws) + kv_plan_bytes(a.c.R));
    const dim3 grid((unsigned)kv_slots(a.c.T, a.c.R, a.G, ROWS), (unsigned)a.c.Hk, ROWS * D / 1024);
    k_attention_join<D, ROWS><<<grid, 256, 0, s>>>(a, plan, parts);
    return hipGetLastError();
}

hipError_t launch_join(const KvAttnArgs& a, int rows, hipStream_t s) {
    switch (a.c.D) {
        case 64: return rows == kRowsTile ? join_of<64, kRowsTile>(a, s) : join_of<64, kTilesTile>(a, s);
        case 128: return rows == kRowsTile ? join_of<128, kRowsTile>(a, s) : join_of<128, kTilesTile>(a, s);
        case 256: return rows == kRowsTile ? join_of<256, kRowsTile>(a, s) : join_of<256, kTilesTile>(a, s);
    }
    return hipErrorInvalidValue;
}

// What a call runs, from the sizes the host knows: query rows of a pair, waves
// of a workgroup that takes a whole pair (0: shares).  Measured, us, the choice
// against the other side (bf16, heads of 128, four query heads a key head unless
// said otherwise; whole pairs of W waves = rows/W, equal shares = rows/0, the
// same for tiles):
//   decode, 8 pairs of 32 blocks    rows/8 14, rows/0 19; of 256: rows/0 21, rows/8 66
//   decode, 512 pairs of 32         rows/4 44, rows/0 48, rows/8 47, rows/1 50
//   decode, 512 pairs of 1 .. 64    rows/4 49, rows/0 53, rows/1 79
//   decode, 1680 pairs of 2         rows/1 17, rows/4 29, rows/0 38
//   decode, 1088 pairs of uneven lengths: rows/2 116, rows/4 107 (equal lengths: 96
//                                   both); the rule sees no lengths and takes rows/2
//   a table of 2048 blocks of which 32 are used: rows/0 18.5 for 8 pairs, 46.5 for 544
//                                   (13.8 and 42.2 with a table of 32)
//   16 x 32 rows on 63 blocks       rows/4 39, tiles/0 51; 13 x 32 on 762: tiles/0 119,
//                                   rows/0 154 (heads of 64: rows/0 61, tiles/0 83)
//   256 x 32 rows on 1 block        rows/1 17, tiles/1 20
//   2000 rows on 8 blocks           rows/2 16, tiles/1 19; 240 on 47: rows/8 19, tiles/0 34
//   8 x 800 rows on 4 blocks        tiles/1 17, rows/1 29, tiles/0 29
//   8000 rows on 32 blocks          tiles/1 57, tiles/0 80, rows/1 132
//   decode, 357 pairs of a table of 159 blocks, 4 seen through a window: rows/4 9,
//                                   rows/0 14
//   16 x 64 rows on 63 blocks, 192 tile pairs: tiles/0 56, tiles/1 98
struct Form {
    int rows, waves;
};

// `blocks`: at most so many of a request's blocks are seen.
Form form_of(int64_t T, int64_t R, int64_t G, int64_t Hk, int D, int64_t blocks) {
    const int64_t rows = T * G;
    const int64_t pairs = kv_slots(T, R, G, kRowsTile) * Hk;
    const int64_t tile_pairs = kv_slots(T, R, G, kTilesTile) * Hk;
    const bool brief = blocks <= 64;
    // Few rows a request, or few tiles, or little to gain from sharing keys
    if (rows <= R * (D == 64 ? 32 : 16) || (brief && (tile_pairs < 256 || rows < R * 48))) {
        if (!brief) return {kRowsTile, 0};
        // As many waves as fit the chip together, and as there are blocks
        int w = 1;
        while (w < 8 && pairs * w * 2 <= (D == 256 ? 1280 : 2560) && w < blocks) w *= 2;
        return {kRowsTile, w};
    }
    return {kTilesTile, tile_pairs >= 384 || blocks <= 16 ? 1 : 0};
}

// The form of a call.  A request's rows, at most T, lie one after the other, so a
// window bounds the blocks that any of them sees.
Form form_of_call(int64_t T, int64_t R, int64_t G, int64_t Hk, int D, int64_t max_blocks, int64_t window) {
    int64_t blocks = max_blocks;
    if (window > 0 && (window + T) / kKvBlock + 2 < blocks) blocks = (window + T) / kKvBlock + 2;
    return form_of(T, R, G, Hk, D, blocks);
}

}  // namespace

// Enough for any window: one that bounds the blocks turns shares into whole pairs,
// never the other way.
size_t kv_attention_workspace(int64_t T, int64_t R, int H, int Hk, int D, int64_t max_blocks) {
    const Form f = form_of(T, R, H / Hk, Hk, D, max_blocks);
    const int64_t grid = f.waves ? 0 : f.rows == kTilesTile ? kTilesShares : kRowsShares;
    return (size_t)(kv_plan_bytes(R) + 2 * grid * f.rows * (D + 3) * 4);
}

hipError_t launch_kv_attention(readme_kv_type kt, const KvAttnArgs& a, hipStream_t s) {
    const Form f = form_of_call(a.c.T, a.c.R, a.G, a.c.Hk, a.c.D, a.c.max_blocks, a.window);
    const hipError_t e = f.rows == kTilesTile ? launch_attention_tiles(kt, a, f.waves == 0, s)
                                              : launch_attention_rows(kt, a, f.waves, s);
    return e != hipSuccess || f.waves ? e : launch_join(a, f.rows, s);
}

}  // namespace readme

// Outside readme.h, for tests: the form that readme_attention_kv takes at these
// sizes, as 256 times the query rows of a pair plus the waves of a workgroup that
// takes a whole pair (1 for tiles), 0 where shares are dealt.
extern "C" int32_t readme_internal_attention_kv_form(int64_t T, int32_t R, int32_t H, int32_t Hk,
                                                     int32_t D, int64_t max_blocks, int64_t window) {
    const readme::Form f = readme::form_of_call(T, R, H / Hk, Hk, D, max_blocks, window);
    return f.rows * 256 + f.waves;
}
