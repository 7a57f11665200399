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
// it keeps its share of the weights and, in the backward pass, of dw and db beside them for all rows
// it visits; the next row's loads are issued before the current row's sums.  Each
// CTA then adds its teams' shares in shared memory and writes one partial row; a second
// kernel adds the partial rows in a fixed order (no atomics: the same bits every time).
#include <cuda_runtime.h>

#include <atomic>

#include "elem.cuh"
#include "gla_internal.h"
#include "tc_ptx.cuh"

namespace gtr {
namespace {

constexpr int kLnThreads = 128;  // CTA of sub-warp and warp teams
constexpr int kLnElems = 16;     // elements of a row a thread holds at most
constexpr int kLnBlockElems = 8; // of a row of up to 8,192 that a whole CTA holds (64 registers a thread)

template <int G> __device__ __forceinline__ float lane_sum(float a) {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
    return a;
}
// Sums over a team of G lanes, or over the CTA (G == 0; every thread calls it, and `buf` is not reused before
// the next barrier of the caller).
template <int G, int N> __device__ __forceinline__ void team_sum(float (&a)[N], float (*buf)[32]) {
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] = lane_sum<G == 0 ? 32 : G>(a[i]);
    if constexpr (G == 0) {
        const int warp = threadIdx.x >> 5, nw = blockDim.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) buf[i][warp] = a[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) a[i] = lane_sum<32>(lane < nw ? buf[i][lane] : 0.f);
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

// A thread's place: its team in the CTA, its rank in the team, the team's threads.
template <int G> struct LnPlace {
    static constexpr int kTeams = G > 0 ? kLnThreads / (G > 0 ? G : 1) : 1;
    int team, rank, width;
    __device__ __forceinline__ LnPlace() {
        if constexpr (G > 0) {
            team = static_cast<int>(threadIdx.x) / G, rank = static_cast<int>(threadIdx.x) % G, width = G;
        } else {
            team = 0, rank = static_cast<int>(threadIdx.x), width = static_cast<int>(blockDim.x);
        }
    }
};
constexpr int ln_max_threads(int g) { return g > 0 ? kLnThreads : 1024; }

// A thread's vectors of the rows to come, NT tensors.  Vectors of 4 bytes and more are copied to the thread's own
// slots of shared memory some rows ahead (nothing but the thread's own wait is between copy and use); single
// 16-bit elements, which cp.async does not copy, go through registers one row ahead.
template <typename E, int VEC, int K, int G, int NT> struct LnAhead {
    using Raw = typename Vec<E, VEC>::raw;
    static constexpr bool kAsync = sizeof(Raw) >= 4;
    // rows held (a CTA team's: what fits 196 KB with two tensors)
    static constexpr int kDepth = !kAsync ? 1 : G > 0 ? 4 : K * VEC * sizeof(E) <= 16 ? 4 : K * VEC * sizeof(E) <= 32 ? (sizeof(E) == 4 ? 3 : 2) : 1;
    static constexpr size_t smem(int threads) { return kAsync ? sizeof(Raw) * kDepth * NT * K * threads : 0; }
    Raw reg[kAsync ? 1 : NT][kAsync ? 1 : K];
    uint8_t *base;
    int slot = 0;

    __device__ __forceinline__ Raw *at(int s, int n, int k) {
        return reinterpret_cast<Raw *>(base) + (static_cast<size_t>((s * NT + n) * K + k) * blockDim.x + threadIdx.x);
    }
    // The next row's vectors (row: its first element per tensor), or nothing.
    __device__ __forceinline__ void fetch(const E *const (&row)[NT], bool live, int rank, int width, int D) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * width + rank) * VEC;
            if (live && c < D) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if constexpr (!kAsync) {
                        reg[n][k] = *reinterpret_cast<const Raw *>(row[n] + c);
                    } else if constexpr (sizeof(Raw) == 16) {
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(at(slot, n, k))),
                                     "l"(row[n] + c)
                                     : "memory");
                    } else {
                        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(ptx::smem_u32(at(slot, n, k))),
                                     "l"(row[n] + c), "n"(sizeof(Raw))
                                     : "memory");
                    }
                }
            }
        }
        if constexpr (kAsync) {
            asm volatile("cp.async.commit_group;" ::: "memory");
            slot = slot + 1 == kDepth ? 0 : slot + 1;
        }
    }
    // Vectors of the oldest row fetched (`fetch` then refills its slot).
    __device__ __forceinline__ void ready() {
        if constexpr (kAsync) asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
    }
    __device__ __forceinline__ Raw get(int n, int k) {
        if constexpr (kAsync) return *at(slot, n, k);
        return reg[n][k];
    }
};

// Columns of thread-vector k: (k width + rank) VEC.
template <typename E, int VEC, int K, int G>
__global__ void __launch_bounds__(ln_max_threads(G), 1) ln_fwd_kernel(const __grid_constant__ LnParams p) {
    using Ahead = LnAhead<E, VEC, K, G, 1>;
    extern __shared__ float4 ln_smem[];
    __shared__ float buf[2][1][32];
    const LnPlace<G> at;
    const float inv = 1.f / static_cast<float>(p.D);
    const long long step = (long long)gridDim.x * at.kTeams;
    Ahead ahead;
    ahead.base = reinterpret_cast<uint8_t *>(ln_smem);
    long long next = (long long)blockIdx.x * at.kTeams + at.team;
    auto fetch = [&] {
        const E *row[1] = {static_cast<const E *>(p.x) + next * p.x_stride};
        ahead.fetch(row, next < p.rows, at.rank, at.width, p.D);
        next += step;
    };
#pragma unroll
    for (int i = 0; i < Ahead::kDepth; ++i) fetch();
    float w[K][VEC], b[K][VEC];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int c = (k * at.width + at.rank) * VEC + i;
            w[k][i] = p.w && c < p.D ? p.w[c] : 1.f;
            b[k][i] = p.b && c < p.D ? p.b[c] : 0.f;
        }
    // whole warps stay in the loop together (their shuffles name all lanes)
    for (long long base = (long long)blockIdx.x * at.kTeams; base < p.rows; base += step) {
        const long long row = base + at.team;
        const bool live = row < p.rows;
        float v[K][VEC], s[1] = {0.f};
        ahead.ready();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (live && (k * at.width + at.rank) * VEC < p.D) {
                Vec<E, VEC>::unpack(ahead.get(0, k), v[k]);
#pragma unroll
                for (int i = 0; i < VEC; ++i) s[0] += v[k][i];
            }
        }
        fetch();
        team_sum<G>(s, buf[0]);
        const float m = s[0] * inv;
        s[0] = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (live && (k * at.width + at.rank) * VEC < p.D) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    v[k][i] -= m;
                    s[0] = fmaf(v[k][i], v[k][i], s[0]);
                }
            }
        team_sum<G>(s, buf[1]);
        const float r = rsqrtf(fmaf(s[0], inv, p.eps));
        if (live && at.rank == 0) {
            if (p.mean) p.mean[row] = m;
            if (p.rstd) p.rstd[row] = r;
        }
        E *y = static_cast<E *>(p.out) + row * p.D;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * at.width + at.rank) * VEC;
            if (live && c < p.D) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[k][i] = fmaf(v[k][i] * r, w[k][i], b[k][i]);
                st_vec<E, VEC>(y + c, v[k]);
            }
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

template <typename E, int VEC, int K, int G>
__global__ void __launch_bounds__(ln_max_threads(G), G > 0 ? 4 : 1) ln_bwd_kernel(const __grid_constant__ LnParams p) {
    using Ahead = LnAhead<E, VEC, K, G, 2>;
    extern __shared__ float4 ln_smem[];
    __shared__ float buf[2][2][32];
    const LnPlace<G> at;
    const float inv = 1.f / static_cast<float>(p.D);
    const long long step = (long long)gridDim.x * at.kTeams;
    Ahead ahead;
    ahead.base = reinterpret_cast<uint8_t *>(ln_smem);
    long long next = (long long)blockIdx.x * at.kTeams + at.team;
    auto fetch = [&] {
        const E *row[2] = {static_cast<const E *>(p.x) + next * p.x_stride, static_cast<const E *>(p.dy) + next * p.dy_stride};
        ahead.fetch(row, next < p.rows, at.rank, at.width, p.D);
        next += step;
    };
#pragma unroll
    for (int i = 0; i < Ahead::kDepth; ++i) fetch();
    float next_m = 0.f, next_r = 0.f;
    auto stats = [&](long long row) {
        if (row < p.rows) next_m = p.mean[row], next_r = p.rstd[row];
    };
    stats((long long)blockIdx.x * at.kTeams + at.team);
    float w[K][VEC], dw[K][VEC] = {}, db[K][VEC] = {};
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int c = (k * at.width + at.rank) * VEC + i;
            w[k][i] = p.w && c < p.D ? p.w[c] : 1.f;
        }
    int flip = 0;
    for (long long base = (long long)blockIdx.x * at.kTeams; base < p.rows; base += step, flip ^= 1) {
        const long long row = base + at.team;
        const bool live = row < p.rows;
        const float m = next_m, r = next_r;
        stats(row + step);
        float h[K][VEC], d[K][VEC], s[2] = {0.f, 0.f};
        ahead.ready();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (live && (k * at.width + at.rank) * VEC < p.D) {
                Vec<E, VEC>::unpack(ahead.get(0, k), h[k]);
                Vec<E, VEC>::unpack(ahead.get(1, k), d[k]);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    h[k][i] = (h[k][i] - m) * r;
                    dw[k][i] = fmaf(d[k][i], h[k][i], dw[k][i]);
                    db[k][i] += d[k][i];
                    d[k][i] *= w[k][i];
                    s[0] += d[k][i];
                    s[1] = fmaf(d[k][i], h[k][i], s[1]);
                }
            }
        }
        fetch();
        team_sum<G>(s, buf[flip]);
        const float c1 = s[0] * inv, c2 = s[1] * inv;
        E *dx = static_cast<E *>(p.out) + row * p.D;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * at.width + at.rank) * VEC;
            if (live && c < p.D) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) h[k][i] = r * (d[k][i] - c1 - h[k][i] * c2);
                st_vec<E, VEC>(dx + c, h[k]);
            }
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    ptx::pdl_launch_dependents();
    if (p.partial == nullptr) return;
    float *share = reinterpret_cast<float *>(ln_smem);  // [teams - 1][2][D], teams of a CTA with several
    if (at.kTeams > 1) {
        __syncthreads();  // the rows ahead are done with
        if (at.team > 0) {
            float *dst = share + (size_t)(at.team - 1) * 2 * p.D;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const int c = (k * at.width + at.rank) * VEC + i;
                    if (c < p.D) dst[c] = dw[k][i], dst[p.D + c] = db[k][i];
                }
        }
        __syncthreads();
        if (at.team > 0) return;
    }
    float *out = p.partial + (size_t)blockIdx.x * 2 * p.D;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int c = (k * at.width + at.rank) * VEC + i;
            if (c < p.D) {
                float a = dw[k][i], b = db[k][i];
                for (int t = 0; t < at.kTeams - 1; ++t) {
                    a += share[(size_t)t * 2 * p.D + c];
                    b += share[(size_t)t * 2 * p.D + p.D + c];
                }
                out[c] = a;
                out[p.D + c] = b;
            }
        }
}

// Sum of the partial rows, columns of dw then db: 8 columns (a 32-byte sector) a CTA, 128 threads down each.
// Launched beside the kernel that writes them, it waits for that one's end.
constexpr int kLnReduceCols = 8, kLnReduceRows = 128;
__global__ void __launch_bounds__(kLnReduceCols * kLnReduceRows)
    ln_reduce_kernel(const float *__restrict__ partial, int nrow, int D, float *dw, float *db) {
    __shared__ float tile[kLnReduceRows][kLnReduceCols + 1];
    const int col = threadIdx.x % kLnReduceCols, row = threadIdx.x / kLnReduceCols, c = blockIdx.x * kLnReduceCols + col;
    ptx::pdl_wait();
    float a = 0.f;
    if (c < 2 * D) {
#pragma unroll 8
        for (int i = row; i < nrow; i += kLnReduceRows) a += partial[(size_t)i * 2 * D + c];
    }
    tile[row][col] = a;
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, o = blockIdx.x * kLnReduceCols + warp;
    if (warp >= kLnReduceCols) return;
    a = 0.f;
#pragma unroll
    for (int i = 0; i < kLnReduceRows / 32; ++i) a += tile[32 * i + lane][warp];
    a = lane_sum<32>(a);
    if (lane == 0) {
        if (o < D) {
            if (dw) dw[o] = a;
        } else if (o < 2 * D) {
            if (db) db[o - D] = a;
        }
    }
}

// How rows are dealt: elements of a load, threads of a row's team (0: the CTA's `threads`), vectors of a thread.
struct LnTeam {
    int vec, g, k, threads;
};
LnTeam ln_team(const LnParams &p, int es) {
    const int v = 16 / es;
    auto fits = [&](int vec) {
        return p.D % vec == 0 && p.x_stride % vec == 0 && (p.dy == nullptr || p.dy_stride % vec == 0);
    };
    const int vec = fits(v) ? v : es == 2 && fits(2) ? 2 : 1;
    const int nv = (p.D + vec - 1) / vec, kmax = kLnElems / vec;
    // 8 lanes read 128 bytes of 16-byte vectors; narrower ones take a warp for that
    if (vec == v && nv <= 8 * kmax) return {vec, 8, (nv + 7) / 8, kLnThreads};
    if (nv <= 32 * kmax) return {vec, 32, (nv + 31) / 32, kLnThreads};
    const int k = p.D <= 1024 * kLnBlockElems ? kLnBlockElems / vec : kmax;
    return {vec, 0, k, ((nv + k - 1) / k + 31) / 32 * 32};
}
int ln_teams(const LnTeam &t) { return t.g > 0 ? kLnThreads / t.g : 1; }

// One instantiation's launch: as many CTAs as the device holds at a time, each walking its rows (the partial
// rows of a backward pass: at most `most`).
template <typename E, int VEC, int K, int G>
cudaError_t ln_run(const LnParams &p, bool bwd, const LnTeam &t, long long most, int *grid, cudaStream_t stream) {
    using Fwd = LnAhead<E, VEC, K, G, 1>;
    using Bwd = LnAhead<E, VEC, K, G, 2>;
    auto *kernel = bwd ? ln_bwd_kernel<E, VEC, K, G> : ln_fwd_kernel<E, VEC, K, G>;
    size_t smem = bwd ? Bwd::smem(t.threads) : Fwd::smem(t.threads);
    if (bwd && p.partial) {
        const size_t share = (size_t)(ln_teams(t) - 1) * 2 * p.D * sizeof(float);  // at most 15 x 2 x 128 floats
        if (share > smem) smem = share;
    }
    int n_sm = 0, dev = 0, per_sm = 0;
    cudaError_t e = sm_count(&n_sm);
    if (e == cudaSuccess) e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    // asked once per device and number of warps
    static std::atomic<int> known[2][64][33] = {};
    std::atomic<int> &fit = known[bwd][dev & 63][t.threads / 32];
    per_sm = fit.load(std::memory_order_relaxed);
    if (per_sm == 0) {
        const int largest = static_cast<int>(bwd ? Bwd::smem(ln_max_threads(G)) : Fwd::smem(ln_max_threads(G)));
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, largest > 48 * 1024 ? largest : 48 * 1024);
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, t.threads, smem);
        if (e != cudaSuccess) return e;
        if (per_sm < 1) return cudaErrorInvalidConfiguration;
        fit.store(per_sm, std::memory_order_relaxed);
    }
    long long n = (p.rows + ln_teams(t) - 1) / ln_teams(t);
    if (n > (long long)n_sm * per_sm) n = (long long)n_sm * per_sm;
    if (n > most) n = most;
    *grid = static_cast<int>(n);
    kernel<<<*grid, t.threads, smem, stream>>>(p);
    return cudaGetLastError();
}
template <typename E, int VEC> cudaError_t ln_run_v(const LnParams &p, bool bwd, const LnTeam &t, long long most, int *grid,
                                                     cudaStream_t s) {
    constexpr int KM = kLnElems / VEC, KH = kLnElems / 2 / VEC;
    static_assert(KH * VEC == kLnBlockElems, "half the elements");
    if (t.g == 0)
        return t.k <= KH ? ln_run<E, VEC, KH, 0>(p, bwd, t, most, grid, s) : ln_run<E, VEC, KM, 0>(p, bwd, t, most, grid, s);
    if constexpr (VEC == 16 / static_cast<int>(sizeof(E))) {
        if (t.g == 8)
            return t.k <= KH ? ln_run<E, VEC, KH, 8>(p, bwd, t, most, grid, s) : ln_run<E, VEC, KM, 8>(p, bwd, t, most, grid, s);
    }
    return t.k <= KH ? ln_run<E, VEC, KH, 32>(p, bwd, t, most, grid, s) : ln_run<E, VEC, KM, 32>(p, bwd, t, most, grid, s);
}
template <typename E> cudaError_t ln_run_e(const LnParams &p, bool bwd, const LnTeam &t, long long most, int *grid,
                                                     cudaStream_t s) {
    if (t.vec == 16 / static_cast<int>(sizeof(E))) return ln_run_v<E, 16 / static_cast<int>(sizeof(E))>(p, bwd, t, most, grid, s);
    if constexpr (sizeof(E) == 2) {
        if (t.vec == 2) return ln_run_v<E, 2>(p, bwd, t, most, grid, s);
    }
    return ln_run_v<E, 1>(p, bwd, t, most, grid, s);
}
cudaError_t ln_launch(const LnParams &p, bool bwd, int dtype, long long most, int *grid, cudaStream_t stream) {
    const LnTeam t = ln_team(p, dtype == 0 ? 4 : 2);
    if (dtype == 0) return ln_run_e<float>(p, bwd, t, most, grid, stream);
    if (dtype == 1) return ln_run_e<__half>(p, bwd, t, most, grid, stream);
    return ln_run_e<__nv_bfloat16>(p, bwd, t, most, grid, stream);
}

// Most partial rows of a backward pass: eight CTAs on each of 152 SMs for rows that a warp holds, fewer the more
// threads a row takes.
long long ln_partial_rows(long long rows, int D) {
    long long cap = 1216LL * 1024 / (D > 1024 ? D : 1024);
    if (cap < 304) cap = 304;
    return rows < cap ? rows : cap;
}

}  // namespace

cudaError_t launch_layernorm(const LnProblem &q, cudaStream_t stream) {
    const LnParams p{q.x, q.x_stride, nullptr, 0, q.weight, q.bias, q.eps, q.rows, q.D, q.out, q.mean, q.rstd, nullptr};
    int grid = 0;
    return ln_launch(p, false, q.dtype, 1LL << 30, &grid, stream);
}

size_t layernorm_bwd_workspace(long long rows, int D) { return (size_t)ln_partial_rows(rows, D) * 2 * D * sizeof(float); }

cudaError_t launch_layernorm_bwd(const LnProblem &q, const void *dy, long long dy_stride, float *dweight, float *dbias,
                                 void *workspace, cudaStream_t stream) {
    const LnParams p{q.x, q.x_stride, dy, dy_stride, q.weight, nullptr, 0.f, q.rows, q.D, q.out, q.mean, q.rstd,
                     (dweight || dbias) ? static_cast<float *>(workspace) : nullptr};
    int grid = 0;
    const cudaError_t e = ln_launch(p, true, q.dtype, ln_partial_rows(q.rows, q.D), &grid, stream);
    if (e != cudaSuccess || !p.partial) return e;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at;
    cfg.gridDim = dim3((2 * q.D + kLnReduceCols - 1) / kLnReduceCols);
    cfg.blockDim = dim3(kLnReduceCols * kLnReduceRows);
    cfg.stream = stream;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, ln_reduce_kernel, static_cast<const float *>(p.partial), grid, q.D, dweight, dbias);
}

}  // namespace gtr
