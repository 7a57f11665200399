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

}  // namespace gtr
