// Which kernel, tile shape and number of splits a matrix product takes.  Host code; no device is asked for anything, so that
// a workspace can be sized where there is none: the kernels are for one device, of 256 compute units.
#pragma once

#include "cgbn_gemm.h"

namespace cgbn {

// number, rows and columns of the tile, wavefronts along each
#define CGBN_TILE_SHAPES(X_) \
    X_(0, 256, 256, 2, 4)    \
    X_(1, 256, 128, 4, 2)    \
    X_(2, 128, 128, 2, 2)    \
    X_(3, 128, 64, 4, 1)     \
    X_(4, 64, 64, 2, 1)

struct GemmPlan {
    int shape, ti, tj, splits, per;
    size_t part_bytes;          // of workspace, 0 where the reduction is not split
};


inline GemmPlan plan_gemm(int elem, bool gated, long long I, long long J, long long R, int segs, int batch)
{
    static const struct { int bi, bj; double rate; } shapes[] = {
        {256, 256, 0.50}, {256, 128, 0.42}, {128, 128, 0.36}, {128, 64, 0.26}, {64, 64, 0.18}};
    const double unit_peak = (elem == 2 ? 2.5e15 : 157e12) / 256;       // operations a second of one compute unit
    const int step = 128 / elem;
    const long long steps = (R + step - 1) / step * segs;
    GemmPlan best{};
    double best_t = 1e30;
    for (int s = 0; s < 5; ++s) {
        const int bj = gated ? shapes[s].bj / 2 : shapes[s].bj;
        const long long ti = (I + shapes[s].bi - 1) / shapes[s].bi, tj = (J + bj - 1) / bj;
        const double t_step = 2.0 * shapes[s].bi * shapes[s].bj * step / (unit_peak * (elem == 2 ? shapes[s].rate : 0.8));
        for (long long want = 1; want <= 256; want = want < 4 ? want + 1 : want + want / 4) {
            if (want > 1 && steps / want < 4) break;
            const long long per = (steps + want - 1) / want, splits = (steps + per - 1) / per;
            const double part = splits > 1 ? (double)splits * batch * (gated ? 2 : 1) * I * J * 4 : 0;
            if (part > 1e9) break;
            const long long groups = ti * tj * batch * splits;
            const double rounds = (double)((groups + 255) / 256);
            const double t = rounds * (per * t_step + 1.5e-6) + (splits > 1 ? 4e-6 + part * 2 / 4e12 : 0);
            if (t < best_t) {
                best_t = t;
                best = GemmPlan{s, (int)ti, (int)tj, (int)splits, (int)per, splits > 1 ? (size_t)part : 0};
            }
        }
    }
    return best;
}

template <typename T, int FORM, bool GATED> hipError_t launch_gemm(const GemmPlan& p, GemmArgs G, hipStream_t st);

}  // namespace cgbn
