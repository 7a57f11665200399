// layernorm.cu -- layer norm over the last dimension and its backward pass.
//
//   m = mean_j x_j,  r = (mean_j (x_j - m)^2 + eps)^{-1/2},  y_j = (x_j - m) r w_j + b_j
//   with xh = (x - m) r and d = dy w:
//   dx = r (d - mean(d) - xh mean(d xh)),  dw = sum over rows of dy xh,  db = sum over rows of dy
//
// Memory-bound: a row is read once into registers (dx's pass: a row of x and of dy), the
// sums run over registers in fp32 (the variance from the centred values, not from a
// difference of moments), and the row is written once.  A row belongs to a team of threads:
// 8 lanes, a warp or a whole CTA, whichever keeps a thread at 16 elements or fewer, so that
// the backward pass can keep its share of dw and db beside them for all rows it visits.  Each
// CTA then adds its teams' shares in shared memory and writes one partial row; a second
// kernel adds the partial rows in a fixed order (no atomics: the same bits every time).
#include <cuda_runtime.h>

#include "elem.cuh"
#include "gla_internal.h"

namespace gtr {
namespace {

constexpr int kLnThreads = 128;      // CTA of sub-warp and warp teams
constexpr int kLnPartialRows = 1216; // most CTAs of a backward pass (partial rows in the workspace)

template <int G> __device__ __forceinline__ float lane_sum(float a) {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
    return a;
}
// Sum over a team of G lanes, or over the CTA (G == 0; every thread calls it, `buf` holds 32 floats
// and is not reused before the next barrier of the caller).
template <int G> __device__ __forceinline__ float team_sum(float a, float *buf) {
    if constexpr (G > 0) {
        return lane_sum<G>(a);
    } else {
        a = lane_sum<32>(a);
        const int warp = threadIdx.x >> 5, nw = blockDim.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0) buf[warp] = a;
        __syncthreads();
        return lane_sum<32>(lane < nw ? buf[lane] : 0.f);
    }
}

struct LnParams {
    const void *x;
    long long x_stride;
    const void *dy;  // backward
    long long dy_stride;
    const float *w, *b;
    float eps;
    long long rows;
    int D;
    void *out;       // y, or dx
    float *mean, *rstd;
    float *partial;  // backward: [gridDim.x][2][D], or null
};

// Columns of thread-vector k: (k G + rank) VEC.
template <typename E, int VEC, int K, int G>
__global__ void __launch_bounds__(G > 0 ? kLnThreads : 1024) ln_fwd_kernel(const __grid_constant__ LnParams p) {
    __shared__ float buf[2][32];
    const int team = G > 0 ? static_cast<int>(threadIdx.x) / (G > 0 ? G : 1) : 0;
    const int rank = G > 0 ? static_cast<int>(threadIdx.x) % (G > 0 ? G : 1) : static_cast<int>(threadIdx.x);
    const int width = G > 0 ? G : static_cast<int>(blockDim.x);
    const int teams = G > 0 ? kLnThreads / (G > 0 ? G : 1) : 1;
    const float inv = 1.f / static_cast<float>(p.D);
    const long long step = (long long)gridDim.x * teams;
    // whole warps stay in the loop together (their shuffles name all lanes)
    for (long long base = (long long)blockIdx.x * teams; base < p.rows; base += step) {
        const long long row = base + team;
        const bool live = row < p.rows;
        const E *x = static_cast<const E *>(p.x) + (live ? row : 0) * p.x_stride;
        float v[K][VEC];
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * width + rank) * VEC;
            if (c < p.D) {
                Vec<E, VEC>::unpack(ld_vec<E, VEC>(x + c), v[k]);
#pragma unroll
                for (int i = 0; i < VEC; ++i) s += v[k][i];
            }
        }
        const float m = team_sum<G>(s, buf[0]) * inv;
        float q = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if ((k * width + rank) * VEC < p.D) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    v[k][i] -= m;
                    q = fmaf(v[k][i], v[k][i], q);
                }
            }
        const float r = rsqrtf(fmaf(team_sum<G>(q, buf[1]), inv, p.eps));
        if (live && rank == 0) {
            if (p.mean) p.mean[row] = m;
            if (p.rstd) p.rstd[row] = r;
        }
        E *y = static_cast<E *>(p.out) + row * p.D;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * width + rank) * VEC;
            if (live && c < p.D) {
                float o[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float h = v[k][i] * r;
                    const float wi = p.w ? p.w[c + i] : 1.f, bi = p.b ? p.b[c + i] : 0.f;
                    o[i] = fmaf(h, wi, bi);
                }
                st_vec<E, VEC>(y + c, o);
            }
        }
    }
}

template <typename E, int VEC, int K, int G>
__global__ void __launch_bounds__(G > 0 ? kLnThreads : 1024) ln_bwd_kernel(const __grid_constant__ LnParams p) {
    __shared__ float buf[2][32];
    extern __shared__ float share[];  // [teams - 1][2][D], teams of a CTA with several
    const int team = G > 0 ? static_cast<int>(threadIdx.x) / (G > 0 ? G : 1) : 0;
    const int rank = G > 0 ? static_cast<int>(threadIdx.x) % (G > 0 ? G : 1) : static_cast<int>(threadIdx.x);
    const int width = G > 0 ? G : static_cast<int>(blockDim.x);
    const int teams = G > 0 ? kLnThreads / (G > 0 ? G : 1) : 1;
    const float inv = 1.f / static_cast<float>(p.D);
    const long long step = (long long)gridDim.x * teams;
    float dw[K][VEC] = {}, db[K][VEC] = {};
    for (long long base = (long long)blockIdx.x * teams; base < p.rows; base += step) {
        const long long row = base + team;
        const bool live = row < p.rows;
        const E *x = static_cast<const E *>(p.x) + (live ? row : 0) * p.x_stride;
        const E *dy = static_cast<const E *>(p.dy) + (live ? row : 0) * p.dy_stride;
        const float m = live ? p.mean[row] : 0.f, r = live ? p.rstd[row] : 0.f;
        float h[K][VEC], d[K][VEC];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * width + rank) * VEC;
            if (live && c < p.D) {
                Vec<E, VEC>::unpack(ld_vec<E, VEC>(x + c), h[k]);
                Vec<E, VEC>::unpack(ld_vec<E, VEC>(dy + c), d[k]);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    h[k][i] = (h[k][i] - m) * r;
                    dw[k][i] = fmaf(d[k][i], h[k][i], dw[k][i]);
                    db[k][i] += d[k][i];
                    if (p.w) d[k][i] *= p.w[c + i];
                    s1 += d[k][i];
                    s2 = fmaf(d[k][i], h[k][i], s2);
                }
            }
        }
        s1 = team_sum<G>(s1, buf[0]) * inv;
        s2 = team_sum<G>(s2, buf[1]) * inv;
        E *dx = static_cast<E *>(p.out) + row * p.D;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * width + rank) * VEC;
            if (live && c < p.D) {
                float o[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) o[i] = r * (d[k][i] - s1 - h[k][i] * s2);
                st_vec<E, VEC>(dx + c, o);
            }
        }
    }
    if (p.partial == nullptr) return;
    if (teams > 1) {
        if (team > 0) {
            float *dst = share + (size_t)(team - 1) * 2 * p.D;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const int c = (k * width + rank) * VEC + i;
                    if (c < p.D) dst[c] = dw[k][i], dst[p.D + c] = db[k][i];
                }
        }
        __syncthreads();
        if (team > 0) return;
    }
    float *out = p.partial + (size_t)blockIdx.x * 2 * p.D;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int c = (k * width + rank) * VEC + i;
            if (c < p.D) {
                float a = dw[k][i], b = db[k][i];
                for (int t = 0; t < teams - 1; ++t) {
                    a += share[(size_t)t * 2 * p.D + c];
                    b += share[(size_t)t * 2 * p.D + p.D + c];
                }
                out[c] = a;
                out[p.D + c] = b;
            }
        }
}

// Sum of the partial rows, columns of dw then db: 32 columns a CTA, 32 threads down each.
__global__ void __launch_bounds__(1024) ln_reduce_kernel(const float *__restrict__ partial, int nrow, int D, float *dw,
                                                         float *db) {
    __shared__ float tile[32][33];
    const int c = blockIdx.x * 32 + threadIdx.x;
    float a = 0.f;
    if (c < 2 * D)
        for (int i = threadIdx.y; i < nrow; i += 32) a += partial[(size_t)i * 2 * D + c];
    tile[threadIdx.y][threadIdx.x] = a;
    __syncthreads();
    a = lane_sum<32>(tile[threadIdx.x][threadIdx.y]);
    const int o = blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x == 0) {
        if (o < D) {
            if (dw) dw[o] = a;
        } else if (o < 2 * D) {
            if (db) db[o - D] = a;
        }
    }
}

// A row's team for D columns in vectors of vec elements: the team's threads (0: the CTA's `threads`)
// and the vectors a thread holds.
struct LnTeam {
    int g, k, threads;
};
LnTeam ln_team(int D, int vec) {
    const int nv = (D + vec - 1) / vec, kmax = 16 / vec;  // 16 elements a thread at most
    if (nv <= 8 * kmax) return {8, (nv + 7) / 8, kLnThreads};
    if (nv <= 32 * kmax) return {32, (nv + 31) / 32, kLnThreads};
    int k = (nv + 255) / 256;  // 256 threads where that is enough
    if (k > kmax) k = kmax;
    return {0, k, ((nv + k - 1) / k + 31) / 32 * 32};
}

int ln_vec(const LnParams &p, int es) {
    const int vec = 16 / es;
    const bool ok = p.D % vec == 0 && p.x_stride % vec == 0 && (p.dy == nullptr || p.dy_stride % vec == 0);
    return ok ? vec : 1;
}

// CTAs of a launch: at most `per_sm` an SM, each walking its rows.
int ln_grid(long long rows, int teams, int n_sm, int per_sm) {
    const long long need = (rows + teams - 1) / teams, cap = (long long)n_sm * per_sm;
    return static_cast<int>(need < cap ? need : cap);
}

template <typename E, int VEC, int K, int G> cudaError_t ln_run(const LnParams &p, bool bwd, const LnTeam &t, int grid,
                                                                  cudaStream_t stream) {
    if (!bwd) {
        ln_fwd_kernel<E, VEC, K, G><<<grid, t.threads, 0, stream>>>(p);
    } else {
        const int teams = G > 0 ? kLnThreads / (G > 0 ? G : 1) : 1;
        const size_t smem = p.partial ? (size_t)(teams - 1) * 2 * p.D * sizeof(float) : 0;  // at most 3 x 2 x 512 floats
        ln_bwd_kernel<E, VEC, K, G><<<grid, t.threads, smem, stream>>>(p);
    }
    return cudaGetLastError();
}
template <typename E, int VEC, int K> cudaError_t ln_run_g(const LnParams &p, bool bwd, const LnTeam &t, int grid,
                                                             cudaStream_t s) {
    if (t.g == 8) return ln_run<E, VEC, K, 8>(p, bwd, t, grid, s);
    if (t.g == 32) return ln_run<E, VEC, K, 32>(p, bwd, t, grid, s);
    return ln_run<E, VEC, K, 0>(p, bwd, t, grid, s);
}
template <typename E> cudaError_t ln_run_e(const LnParams &p, bool bwd, int vec, const LnTeam &t, int grid, cudaStream_t s) {
    constexpr int V = 16 / static_cast<int>(sizeof(E));
    if (vec == V) {
        if (t.k <= 1) return ln_run_g<E, V, 1>(p, bwd, t, grid, s);
        if (t.k <= 2) return ln_run_g<E, V, 2>(p, bwd, t, grid, s);
        return ln_run_g<E, V, 16 / V>(p, bwd, t, grid, s);
    }
    if (t.k <= 4) return ln_run_g<E, 1, 4>(p, bwd, t, grid, s);
    return ln_run_g<E, 1, 16>(p, bwd, t, grid, s);
}

cudaError_t ln_launch(const LnParams &p, bool bwd, int dtype, int grid, cudaStream_t stream) {
    const int es = dtype == 0 ? 4 : 2, vec = ln_vec(p, es);
    const LnTeam t = ln_team(p.D, vec);
    if (dtype == 0) return ln_run_e<float>(p, bwd, vec, t, grid, stream);
    if (dtype == 1) return ln_run_e<__half>(p, bwd, vec, t, grid, stream);
    return ln_run_e<__nv_bfloat16>(p, bwd, vec, t, grid, stream);
}

int ln_teams(const LnTeam &t) { return t.g > 0 ? kLnThreads / t.g : 1; }

}  // namespace

cudaError_t launch_layernorm(const LnProblem &q, cudaStream_t stream) {
    int n_sm = 0;
    cudaError_t e = sm_count(&n_sm);
    if (e != cudaSuccess) return e;
    LnParams p{q.x, q.x_stride, nullptr, 0, q.weight, q.bias, q.eps, q.rows, q.D, q.out, q.mean, q.rstd, nullptr};
    const LnTeam t = ln_team(p.D, ln_vec(p, q.dtype == 0 ? 4 : 2));
    return ln_launch(p, false, q.dtype, ln_grid(q.rows, ln_teams(t), n_sm, 16), stream);
}

size_t layernorm_bwd_workspace(long long rows, int D) {
    const long long n = rows < kLnPartialRows ? rows : kLnPartialRows;
    return (size_t)n * 2 * D * sizeof(float);
}

cudaError_t launch_layernorm_bwd(const LnProblem &q, const void *dy, long long dy_stride, float *dweight, float *dbias,
                                 void *workspace, cudaStream_t stream) {
    int n_sm = 0;
    cudaError_t e = sm_count(&n_sm);
    if (e != cudaSuccess) return e;
    LnParams p{q.x, q.x_stride, dy, dy_stride, q.weight, nullptr, 0.f, q.rows, q.D, q.out, q.mean, q.rstd,
               (dweight || dbias) ? static_cast<float *>(workspace) : nullptr};
    const LnTeam t = ln_team(p.D, ln_vec(p, q.dtype == 0 ? 4 : 2));
    int grid = ln_grid(q.rows, ln_teams(t), n_sm, t.g > 0 ? 4 : 2);
    if (grid > kLnPartialRows) grid = kLnPartialRows;
    if ((e = ln_launch(p, true, q.dtype, grid, stream)) != cudaSuccess) return e;
    if (!p.partial) return cudaSuccess;
    ln_reduce_kernel<<<(2 * q.D + 31) / 32, dim3(32, 32), 0, stream>>>(p.partial, grid, q.D, dweight, dbias);
    return cudaGetLastError();
}

}  // namespace gtr
