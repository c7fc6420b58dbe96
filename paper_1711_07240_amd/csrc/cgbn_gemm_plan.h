// Which tile shape and how many splits of the reduction a matrix product takes.  Host code; no device is asked for anything, so
// that a workspace can be sized where there is none: the kernels are for one device, of 256 compute units.
#pragma once

#include "cgbn_gemm.h"

namespace cgbn {

// number, rows and columns of the tile, wavefronts along each
#define CGBN_TILE_SHAPES(X_) \
    X_(0, 256, 256, 2, 2)    \
    CGBN_TILE_SHAPES_FLOAT(X_)
// (float has two sets of accumulators)
#define CGBN_TILE_SHAPES_FLOAT(X_) \
    X_(1, 128, 128, 2, 2)          \
    X_(2, 128, 64, 4, 1)           \
    X_(3, 64, 64, 2, 1)

// of a launch's axis (of more the runtime starts some, without an error)
constexpr double kMaxThreads = 4294967295.;

struct GemmPlan {
    int shape, elem, ti, tj, splits, per;
    size_t part_bytes;          // of workspace, 0 where the reduction is not split
    double groups;              // workgroups
    double work, besides;       // seconds that a full compute unit spends on one's products, and on its loads and stores
    double join;                // seconds for joining the splits
};

// The shapes' rates, in operations a second of the whole device with the compute units full: as measured on 8192 x 8192 x 8192
// (float: 8192 x 8192 x 2048).  Where a vector unit holds few wavefronts, their waits show: the fraction of the rate with one and with two of
// them; `start`, their prologue's time.
struct TileShape {
    int bi, bj, waves;
    int fit;                    // workgroups that a compute unit holds
    double start;
    struct { double full, one, two; } rate[2];          // bfloat16, float
};
inline const TileShape& tile_shape(int s)
{
    static const TileShape shapes[] = {{256, 256, 4, 1, 7e-6, {{1450e12, 1., 1.}, {0., 0., 0.}}},
                                       {128, 128, 4, 2, 0.8e-6, {{1170e12, 0.68, 1.}, {198e12, 0.72, 1.}}},
                                       {128, 64, 4, 3, 0.5e-6, {{900e12, 0.55, 0.85}, {162e12, 0.5, 0.7}}},
                                       {64, 64, 2, 5, 0.3e-6, {{690e12, 0.85, 0.95}, {153e12, 0.47, 0.75}}}};
    return shapes[s];
}
constexpr int kTileShapes = 4;

// Forward products of bfloat16 with short reductions and many tiles take a tile of their own instead of 128 x 128 or 256 x 256: two
// workgroups just fit the LDS of a compute unit, so that one multiplies while the other's results travel, and they read a fifth less from LDS
// than with 128 x 128.  Microseconds without it and with it, without residual and with one:
//   67200 x 64 x 1024    57, 50; 78, 75      67200 x 512 x 1024   119, 104; 118, 113     67200 x 1024 x 1024   184, 160; 187, 169
//   16384 x 64 x 4096    54, 50; 94, 73      16384 x 512 x 4096   103, 90; 194, 113      16384 x 2048 x 4096   -; 320, 273
// Not where rows of the result do not start on lines of 128 bytes and there is little else to do: 9000 x 64 x 9000 85, 94 and 128, 132;
// 9000 x 1000 x 9000 227, 210 and 255, 247.  Longer reductions are 256 x 256's: 8192 x 8192 x 8192 870 with this tile, 772.
constexpr int kShortI = 192, kShortJ = 128;
inline bool short_shape(int shape, int splits, long long I, long long J, long long R, bool residual)
{
    return shape <= 1 && splits == 1 && R <= (residual ? 2048 : 1024) && (R >= 512 || J % 64 == 0) &&
           (I + kShortI - 1) / kShortI * ((J + kShortJ - 1) / kShortJ) >= 2048 &&
           (double)((I + kShortI - 1) / kShortI * ((J + kShortJ - 1) / kShortJ)) * 4 * kWave <= kMaxThreads;
}

// the plan with one shape and one number of splits; false: more than can be
inline bool plan_with(int shape, long long want, int elem, bool gated, long long I, long long J, long long R, int segs, int batch, GemmPlan* p)
{
    const TileShape& t = tile_shape(shape);
    if (t.rate[elem == 4].full == 0.) return false;
    const int step = 128 / elem, bj = gated ? t.bj / 2 : t.bj;
    const long long steps = (R + step - 1) / step * segs, per = (steps + want - 1) / want, splits = (steps + per - 1) / per;
    const double part = splits > 1 ? (double)splits * batch * (gated ? 2 : 1) * I * J * 4 : 0;
    const long long ti = (I + t.bi - 1) / t.bi, tj = (J + bj - 1) / bj;
    if (part > 1e9 || (double)ti * tj * splits * batch * t.waves * kWave > kMaxThreads) return false;
    *p = GemmPlan{shape, elem, (int)ti, (int)tj, (int)splits, (int)per, (size_t)part, (double)ti * tj * splits * batch, 0, 0, 0};
    // (what a workgroup does besides: its first loads' way, and its rows of A, which it shares with the tiles beside it, and its
    // results, at the rate of memory)
    const double bytes = (double)t.bi * per * 128 / (double)(tj < 8 ? tj : 8) + (double)t.bi * bj * (gated ? 2 : 1) * (splits > 1 ? 4 : elem * 1.25);
    p->besides = t.start + bytes / (5e12 / 256);
    p->work = per * 2. * t.bi * t.bj * step / (t.rate[elem == 4].full / 256);
    // (written and read back from the caches.  Of 282 forward products of 33 to 2048 rows, timed with every shape and split, those that
    // this model takes are 4% off the best on the mean where it was chosen and 6% elsewhere, 5% and 7% with half of this rate; with 6e12
    // 3000 x 768 x 768 float has dW split for nothing, 83 us for 69)
    p->join = splits > 1 ? 5e-6 + part / 4e12 : 0;
    return true;
}

// seconds that a compute unit spends on one workgroup of a launch of `groups` of them
inline double cost_of(const GemmPlan& p, double groups)
{
    const TileShape& t = tile_shape(p.shape);
    // wavefronts of a compute unit's workgroups, dealt over its four vector units: the busiest has `deep` of them
    const double waves = (double)((long long)((groups + 255) / 256)) * t.waves / 4, deep = (double)(long long)(waves + 0.75);
    const auto& rate = t.rate[p.elem == 4];
    return p.work / (waves / deep * (deep <= 1 ? rate.one : deep <= 2 ? rate.two : 1.)) + p.besides;
}

template <typename F> inline void each_split(long long steps, F f)
{
    // (a split of fewer than four steps is all prologue; powers of two fill 256 compute units evenly)
    for (long long want = 1, by = 1; want == 1 || (want <= 256 && steps / want >= 4); want += by, by = want >= 8 * by ? 2 * by : by)
        if (!f(want)) break;
}

// the seconds of a product by itself: rounds of workgroups
inline double time_alone(const GemmPlan& p) { return (double)(long long)((p.groups + 255) / 256) * cost_of(p, p.groups) + p.join; }

inline GemmPlan plan_shape(int shape, int elem, bool gated, long long I, long long J, long long R, int segs, int batch)
{
    const int step = 128 / elem;
    GemmPlan best{}, p;
    each_split((R + step - 1) / step * segs, [&](long long want) {
        if (!plan_with(shape, want, elem, gated, I, J, R, segs, batch, &p)) return false;
        if (best.ti == 0 || time_alone(p) < time_alone(best)) best = p;
        return true;
    });
    return best;
}

inline GemmPlan plan_gemm(int elem, bool gated, long long I, long long J, long long R, int segs, int batch)
{
    GemmPlan best{};
    for (int s = 0; s < kTileShapes; ++s) {
        const GemmPlan p = plan_shape(s, elem, gated, I, J, R, segs, batch);
        if (p.ti && (best.ti == 0 || time_alone(p) < time_alone(best))) best = p;
    }
    return best;
}

// dx [M][K] = dz [M][N] W and dW [N][K] = dz^T x, `pairs` of them, in one launch and with one shape
inline void plan_two(int elem, long long M, int N, int K, int pairs, GemmPlan* dx, GemmPlan* dw)
{
    const int step = 128 / elem;
    double best = 0;
    dx->ti = 0;
    for (int s = 0; s < kTileShapes; ++s) {
        GemmPlan w[2], x;
        w[0] = plan_shape(s, elem, false, N, K, M, 1, pairs);
        if (!w[0].ti || !plan_with(s, 1, elem, false, N, K, M, 1, pairs, &w[1])) continue;
        each_split((N + step - 1) / step * pairs, [&](long long want) {
            if (!plan_with(s, want, elem, false, M, K, N, pairs, 1, &x)) return false;
            for (int b = 0; b < 2; ++b) {
                const double groups = x.groups + w[b].groups;
                if (groups * tile_shape(s).waves * kWave > kMaxThreads) continue;
                const double cx = cost_of(x, groups), cw = cost_of(w[b], groups);
                // A unit takes the next workgroup when it is done with one: the last to be started end half of one's time after
                // the average.  One that shares its unit takes as many times longer: a long one, dx unsplit for few rows, is then
                // what the launch waits for (64 x 4096 x 4096 float 190 us with dx in 64 workgroups among 4096 of dW, 67 split).
                const double most = groups / 256 < tile_shape(s).fit ? groups / 256 : tile_shape(s).fit, share = most > 1 ? most : 1;
                double t = (x.groups * cx + w[b].groups * cw) / 256 + 0.5 * cw;
                if (t < cx * share) t = cx * share;
                if (t < cw * share) t = cw * share;
                t += x.join + w[b].join;
                if (dx->ti == 0 || t < best) {
                    best = t;
                    *dx = x;
                    *dw = w[b];
                }
            }
            return true;
        });
    }
}

// the sums of a split forward product joined, the epilogue
template <typename T, bool GATED> hipError_t launch_join(const GemmArgs& G, hipStream_t st);
template <typename T, int FORM, bool GATED> hipError_t launch_gemm(const GemmPlan& p, GemmArgs G, hipStream_t st);
// both products of a backward pass in one launch
template <typename T> hipError_t launch_two(const GemmPlan& px, GemmArgs X, const GemmPlan& pw, GemmArgs W, hipStream_t st);

}  // namespace cgbn
