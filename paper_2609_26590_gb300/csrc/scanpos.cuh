// scanpos.cuh -- the spatial token behind a scan position, and the walk to the next ones.
#pragma once

#include "fastdiv.cuh"

namespace gtr {

// Sec. 3.1, directional scanning: position s of the four raster orders (gtr_scan_t) on a grid of
// gh x gw tokens stored row-major.
struct ScanGrid {
    FastDiv gh;
    int gw, T, order;
};
inline ScanGrid make_scan_grid(int grid_h, int grid_w, int order) {
    return ScanGrid{make_fastdiv(grid_h), grid_w, grid_h * grid_w, order};
}
struct ScanPos {
    int t, row;  // token; grid row (column orders)
    __device__ __forceinline__ void set(const ScanGrid &g, int s) {
        const int u = (g.order & 1) ? g.T - 1 - s : s;
        if (g.order & 2) {
            const int col = fdiv(u, g.gh);
            row = u - col * g.gh.d;
            t = row * g.gw + col;
        } else {
            row = 0;
            t = u;
        }
    }
    __device__ __forceinline__ void next(const ScanGrid &g) {
        if (!(g.order & 2)) {
            t += (g.order & 1) ? -1 : 1;
        } else if (!(g.order & 1)) {
            t += g.gw;
            if (++row == g.gh.d) t += 1 - g.T, row = 0;  // T = gh gw: back to row 0, one column on
        } else {
            t -= g.gw;
            if (--row < 0) t += g.T - 1, row = g.gh.d - 1;
        }
    }
};

// The same walk as an address: `stride` elements a token.
template <typename P> struct ScanWalk {
    P *at;
    long long on, over;  // to the next position, and from the last one of a column (column orders)
    int left, run;       // positions before that
    __device__ __forceinline__ ScanWalk(const ScanGrid &g, const ScanPos &pos, P *base, long long stride) {
        at = base + pos.t * stride;
        const long long one = (g.order & 1) ? -1 : 1;
        if (g.order & 2) {
            on = one * g.gw * stride;
            over = one * (1 - static_cast<long long>(g.T - g.gw)) * stride;
            left = (g.order & 1) ? pos.row : g.gh.d - 1 - pos.row;
            run = g.gh.d - 1;
        } else {
            on = over = one * stride;
            left = run = 0x7fffffff;
        }
    }
    __device__ __forceinline__ void next() {
        at += left > 0 ? on : over;
        left = left > 0 ? left - 1 : run;
    }
};

}  // namespace gtr
