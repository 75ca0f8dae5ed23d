// readme_rotary: rows turned by their positions (rotary.hpp has the mathematics).
//
// A thread has one chunk of sixteen dims of one token: its eight sines and
// cosines stay in registers while it goes over every G-th head, so that G head
// groups of a token compute them G times and no more.  Bound by the rows' stream:
// 8192 tokens of 40 heads of 128 in bf16, 168 MB, 35 us, 4.8 TB/s (a large copy 5.0);
// 3001 of 12 heads of 80 in fp32, 23 MB, 8.4; a token of 8 heads 2.8, the launch.
#include "rotary.hpp"

namespace readme {

namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;  // heads whose loads are issued before the first store

template <int DT>
__global__ __launch_bounds__(kThreads) void k_rotary(int64_t T, int H, int D, int groups, RotaryArgs a,
                                                     const void* x, int64_t ld_x, void* y,
                                                     int64_t ld_y) {
    constexpr int N = DT == README_F32 ? 2 : 1;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int chunks = D / 16;
    const int64_t tg = i / chunks;
    const int ch = (int)(i - tg * chunks);
    const int64_t t = tg / groups;
    if (t >= T) return;
    const int g = (int)(tg - t * groups);
    const Chunk k = chunk_of(ch, a.rot, a.layout);
    if (!k.turns && x == y) return;
    uint4 ra[kBatch][N], rb[kBatch][N];
    auto load = [&](int h0) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int h = h0 + j * groups;
            if (h >= H) break;
            const int64_t at = t * ld_x + (int64_t)h * D;
            load8<DT>(x, at + k.a, ra[j]);
            load8<DT>(x, at + k.b, rb[j]);
        }
    };
    load(g);  // on their way while the angles are computed
    Turn turns[8];
    if (k.turns) {
        const double pos = (double)a.pos[t];
        const float sign = a.inverse ? -1.0f : 1.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) turns[e] = turn_of(pos, a.freqs[8 * ch + e], a.amplitude, sign);
    }
    for (int h0 = g; h0 < H; h0 += kBatch * groups) {
        if (h0 != g) load(h0);
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int h = h0 + j * groups;
            if (h >= H) break;
            const int64_t at = t * ld_y + (int64_t)h * D;
            if (k.turns) {
                float v[16];
                widen8<DT>(ra[j], v);
                widen8<DT>(rb[j], v + 8);
                turn_chunk(turns, a.layout, v);
                narrow8<DT>(v, ra[j]);
                narrow8<DT>(v + 8, rb[j]);
            }
            store8<DT>(y, at + k.a, ra[j]);
            store8<DT>(y, at + k.b, rb[j]);
        }
    }
}

}  // namespace

hipError_t launch_rotary(readme_dtype dt, int64_t T, int H, int D, const RotaryArgs& a, const void* x,
                         int64_t ld_x, void* y, int64_t ld_y, hipStream_t s) {
    // Head groups of a token until the threads fill the chip (16 waves a CU).  Against
    // one group, us: a token of 71 heads 3.1 for 22.3, 512 of 32 4.2 for 11.5, 8192 of
    // 40 34.9 for 37.2; 8 and 32 waves a CU: 37.7 and 36.0 for the last.
    const int64_t one = T * (D / 16);
    int64_t groups = ceil_div(256 * 16 * 64, one);
    groups = groups < 1 ? 1 : (groups > H ? H : groups);
    const int64_t grid = ceil_div(one * groups, kThreads);
    if (dt == README_F32)
        k_rotary<README_F32><<<(unsigned)grid, kThreads, 0, s>>>(T, H, D, (int)groups, a, x, ld_x, y, ld_y);
    else
        k_rotary<README_BF16><<<(unsigned)grid, kThreads, 0, s>>>(T, H, D, (int)groups, a, x, ld_x, y, ld_y);
    return hipGetLastError();
}

}  // namespace readme
