// conv.cu -- short causal depthwise convolution along a scan order, optionally followed by SiLU:
//   a_s = b + sum_{j < W} w_j x_{s - W + 1 + j},  y_s = SiLU(a_s)
// with the W - 1 inputs before the sequence zero or given, and the last W - 1 inputs returned as
// the state from which single tokens go on.
//
// Memory-bound: each input is read once (and W - 1 again at the start of a strip, from L2), each
// output written once.  A thread owns four channels (two or one where the
// alignment does not allow that) and walks a strip of scan positions with the last W inputs
// in registers; the scan order is in the walk's addresses.
//
// Measured on a GB300: 32 x 40 x 40 x 768 bf16, column order, 30.9 us (5.1 TB/s of the bytes that have to move, 75 % of
// the measured copy); bound by the copies in flight and the issue of SiLU's instructions together.  Loads in
// registers, four positions ahead: 60 us; addresses formed from the position for each token: 48 us.  Single tokens
// of 256 x 1,536 fp16: 3.3 us.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>

#include "elem.cuh"
#include "gla_internal.h"
#include "scanpos.cuh"
#include "tc_ptx.cuh"

namespace gtr {
namespace {

constexpr int kConvThreads = 256;
constexpr int kConvStrip = 128; // most scan positions a thread walks
constexpr int kConvBatch = 4;   // positions loaded at a time
constexpr int kConvDepth = 4;   // batches in flight

struct ConvParams {
    const void *x;
    long long x_stride;
    const float *w, *b;
    const void *init;
    void *out, *state;
    ScanGrid grid;
    int B, E, silu, strip, strips;  // positions of a strip, strips of a sequence
    long long items;  // B * strips
};

// The taps of VEC channels: VEC W consecutive floats, in 16-byte loads where they start on such.
template <int VEC, int W> __device__ __forceinline__ void load_taps(const float *w, float (&tap)[W][VEC]) {
    if (VEC * W % 4 == 0 && (reinterpret_cast<uintptr_t>(w) & 15u) == 0) {
#pragma unroll
        for (int i = 0; i < VEC * W / 4; ++i) {
            const float4 f = reinterpret_cast<const float4 *>(w)[i];
            const float v[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) tap[(4 * i + k) % W][(4 * i + k) / W] = v[k];
        }
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j) tap[j][i] = w[i * W + j];
    }
}

template <typename E, int VEC, int W>
__global__ void __launch_bounds__(kConvThreads, 3) conv_kernel(const __grid_constant__ ConvParams p) {
    using Raw = typename Vec<E, VEC>::raw;
    const long long item = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    const int c = (blockIdx.y * blockDim.x + threadIdx.x) * VEC;
    if (item >= p.items || c >= p.E) return;
    const int b = static_cast<int>(item / p.strips), strip = static_cast<int>(item - (long long)b * p.strips);
    const int T = p.grid.T, s0 = strip * p.strip, s1 = T - s0 < p.strip ? T : s0 + p.strip;
    const E *x = static_cast<const E *>(p.x) + (long long)b * T * p.x_stride + c;
    const E *init = p.init ? static_cast<const E *>(p.init) + (long long)b * (W - 1) * p.E + c : nullptr;
    E *out = static_cast<E *>(p.out) + (long long)b * T * p.E + c;
    // The positions ahead: copied to the thread's own slots of shared memory kConvDepth batches ahead (nothing but
    // its own wait is between copy and use); single 16-bit elements, which cp.async does not copy, wait in
    // registers, one batch ahead.
    constexpr bool ASYNC = sizeof(Raw) >= 4;
    extern __shared__ uint4 conv_smem[];
    const uint32_t pitch = static_cast<uint32_t>(sizeof(Raw)) * blockDim.x * blockDim.y;  // between a thread's slots
    const uint32_t slots = ptx::smem_u32(conv_smem) + static_cast<uint32_t>(sizeof(Raw)) * (threadIdx.y * blockDim.x + threadIdx.x);
    Raw in[kConvBatch];
    ScanPos start;
    start.set(p.grid, s0);
    ScanWalk<const E> ahead(p.grid, start, x, p.x_stride);
    ScanWalk<E> to(p.grid, start, out, p.E);
    int fetched = s0;
    uint32_t slot = slots;
    auto fetch = [&] {
#pragma unroll
        for (int k = 0; k < kConvBatch; ++k) {
            const bool live = fetched + k < s1;
            if constexpr (!ASYNC) {
                if (live) in[k] = *reinterpret_cast<const Raw *>(ahead.at);
            } else if constexpr (sizeof(Raw) == 16) {
                asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p cp.async.cg.shared.global [%0], [%1], 16;\n\t}" ::"r"(
                                 slot + k * pitch),
                             "l"(ahead.at), "r"(static_cast<uint32_t>(live))
                             : "memory");
            } else {
                asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p cp.async.ca.shared.global [%0], [%1], %3;\n\t}" ::"r"(
                                 slot + k * pitch),
                             "l"(ahead.at), "r"(static_cast<uint32_t>(live)), "n"(sizeof(Raw))
                             : "memory");
            }
            ahead.next();
        }
        fetched += kConvBatch;
        if constexpr (ASYNC) {
            asm volatile("cp.async.commit_group;" ::: "memory");
            slot += kConvBatch * pitch;
            if (slot == slots + kConvDepth * kConvBatch * pitch) slot = slots;
        }
    };
#pragma unroll
    for (int i = 0; i < (ASYNC ? kConvDepth : 1); ++i) fetch();
    // taps, bias and the window of inputs s - W + 1 .. s, as packed pairs (a single channel: the upper half unused)
    constexpr int P = (VEC + 1) / 2;
    f2 w[W][P], bias[P], win[W][P];
    auto pairs = [](const float (&f)[VEC], f2(&g)[P]) {
#pragma unroll
        for (int i = 0; i < P; ++i) g[i] = pack2(f[2 * i], 2 * i + 1 < VEC ? f[(2 * i + 1) % VEC] : 0.f);
    };
    auto widen = [&](const Raw &r, f2(&g)[P]) {
        float f[VEC];
        Vec<E, VEC>::unpack(r, f);
        pairs(f, g);
    };
    {
        float taps[W][VEC], f[VEC];
        load_taps<VEC, W>(p.w + (long long)c * W, taps);
#pragma unroll
        for (int j = 0; j < W; ++j) pairs(taps[j], w[j]);
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[i] = p.b ? p.b[c + i] : 0.f;
        pairs(f, bias);
    }
#pragma unroll
    for (int j = 1; j < W; ++j) {  // inputs s0 - W + j
        const int s = s0 - W + j;
#pragma unroll
        for (int i = 0; i < P; ++i) win[j][i] = 0;
        if (s >= 0) {
            ScanPos q;
            q.set(p.grid, s);
            widen(ld_vec<E, VEC>(x + (long long)q.t * p.x_stride), win[j]);
        } else if (init) {
            widen(ld_vec<E, VEC>(init + (long long)(s + W - 1) * p.E), win[j]);
        }
    }
    auto narrow = [](const f2(&g)[P]) {
        float f[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float2 a = unpack2(g[i / 2]);
            f[i] = i % 2 ? a.y : a.x;
        }
        return Vec<E, VEC>::pack(f);
    };
    auto output = [&](const Raw &r, f2(&a)[P]) {  // takes in one input: its sum
#pragma unroll
        for (int j = 0; j + 1 < W; ++j)
#pragma unroll
            for (int i = 0; i < P; ++i) win[j][i] = win[j + 1][i];
        widen(r, win[W - 1]);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            a[i] = bias[i];
#pragma unroll
            for (int j = 0; j < W; ++j) a[i] = fma2(w[j][i], win[j][i], a[i]);
        }
    };
    for (int s = s0; s < s1; s += kConvBatch) {
        Raw now[kConvBatch];
        if constexpr (ASYNC) asm volatile("cp.async.wait_group %0;" ::"n"(kConvDepth - 1) : "memory");
#pragma unroll
        for (int k = 0; k < kConvBatch; ++k) {
            if constexpr (ASYNC)
                now[k] = *reinterpret_cast<const Raw *>(reinterpret_cast<const uint8_t *>(conv_smem) +
                                                        (slot - ptx::smem_u32(conv_smem) + k * pitch));  // (what no copy wrote is not used)
            else
                now[k] = in[k];
        }
        fetch();
        if (s + kConvBatch <= s1) {
            f2 a[kConvBatch][P];
#pragma unroll
            for (int k = 0; k < kConvBatch; ++k) output(now[k], a[k]);
            if (p.silu) {
#pragma unroll
                for (int k = 0; k < kConvBatch; ++k)
#pragma unroll
                    for (int i = 0; i < P; ++i) a[k][i] = silu_pair<E>(a[k][i]);
            }
#pragma unroll
            for (int k = 0; k < kConvBatch; ++k) {
                *reinterpret_cast<Raw *>(to.at) = narrow(a[k]);
                to.next();
            }
        } else {  // the last positions of a sequence
#pragma unroll
            for (int k = 0; k + 1 < kConvBatch; ++k) {
                if (s + k < s1) {
                    f2 a[P];
                    output(now[k], a);
                    if (p.silu) {
#pragma unroll
                        for (int i = 0; i < P; ++i) a[i] = silu_pair<E>(a[i]);
                    }
                    *reinterpret_cast<Raw *>(to.at) = narrow(a);
                    to.next();
                }
            }
        }
    }
    if constexpr (ASYNC) asm volatile("cp.async.wait_all;" ::: "memory");
    if (p.state && s1 == T) {  // the window's last W - 1 inputs (exact: they are stored values)
        E *st = static_cast<E *>(p.state) + (long long)b * (W - 1) * p.E + c;
#pragma unroll
        for (int j = 0; j + 1 < W; ++j) *reinterpret_cast<Raw *>(st + (long long)j * p.E) = narrow(win[j + 1]);
    }
}

// One token of every sequence: reads the state and the token, writes the output and the moved state
// (which may be the state's own memory: a thread reads its channels before it writes them).
template <typename E, int VEC, int W>
__global__ void __launch_bounds__(kConvThreads) conv_step_kernel(const __grid_constant__ ConvParams p) {
    const int b = blockIdx.x * blockDim.y + threadIdx.y;
    const int c = (blockIdx.y * blockDim.x + threadIdx.x) * VEC;
    if (b >= p.B || c >= p.E) return;
    typename Vec<E, VEC>::raw in[W];
    const E *init = static_cast<const E *>(p.init) + (long long)b * (W - 1) * p.E + c;
#pragma unroll
    for (int j = 0; j + 1 < W; ++j) in[j] = ld_vec<E, VEC>(init + (long long)j * p.E);
    in[W - 1] = ld_vec<E, VEC>(static_cast<const E *>(p.x) + (long long)b * p.x_stride + c);
    float a[VEC], w[W][VEC];
    load_taps<VEC, W>(p.w + (long long)c * W, w);
#pragma unroll
    for (int i = 0; i < VEC; ++i) a[i] = p.b ? p.b[c + i] : 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) {
        float f[VEC];
        Vec<E, VEC>::unpack(in[j], f);
#pragma unroll
        for (int i = 0; i < VEC; ++i) a[i] = fmaf(w[j][i], f[i], a[i]);
    }
    if (p.silu) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) a[i] = silu<E>(a[i]);
    }
    st_vec<E, VEC>(static_cast<E *>(p.out) + (long long)b * p.E + c, a);
    E *st = static_cast<E *>(p.state) + (long long)b * (W - 1) * p.E + c;
#pragma unroll
    for (int j = 0; j + 1 < W; ++j)
        *reinterpret_cast<typename Vec<E, VEC>::raw *>(st + (long long)j * p.E) = in[j + 1];
}

template <typename E, int VEC> size_t conv_smem_bytes(int threads) {  // at most 64 KB
    const size_t raw = sizeof(typename Vec<E, VEC>::raw);
    return raw >= 4 ? raw * kConvBatch * kConvDepth * threads : 0;
}

// CTAs of one instantiation that an SM holds, asked once per device and number of warps.
template <typename E, int VEC, int W> cudaError_t conv_fit(int threads, int *per_sm) {
    static std::atomic<int> known[64][kConvThreads / 32 + 1] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const int warps = (threads + 31) / 32;
    std::atomic<int> &fit = known[dev & 63][warps];
    *per_sm = fit.load(std::memory_order_relaxed);
    if (*per_sm > 0) return cudaSuccess;
    auto *kernel = conv_kernel<E, VEC, W>;
    const size_t most = conv_smem_bytes<E, VEC>(kConvThreads);
    if (most > 48 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(most));
    if (e == cudaSuccess)
        e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(per_sm, kernel, 32 * warps, conv_smem_bytes<E, VEC>(32 * warps));
    if (e != cudaSuccess) return e;
    if (*per_sm < 1) return cudaErrorInvalidConfiguration;
    fit.store(*per_sm, std::memory_order_relaxed);
    return cudaSuccess;
}

// The scan positions of a strip, by what the busiest SM takes for its rounds of CTAs: a start of 13 positions' latency
// (taps, the window, the first copies), then each position that latency or the CTAs' bytes, whichever is more
// (cta_bytes: warps x bytes a lane; 57 of them take one latency).  Fitted to 13 problems at 20 lengths on a GB300.  In us,
// against strips of 32 halved until there were 1,024 threads an SM: bf16 32 x 1,600 x 768 30.9 (35.4), 128 x 1,600 x 768
// 103 (119); fp32 32 x 1,600 x 768 62 (66.7); fp16 4 x 1,600 x 768 8.7 (12.3), 4 x 400 x 1,536 5.8 (7.2), 300 x 49 x 768
// 11.6 (15.0), 16 x 784 x 500 11.0 (11.3); slower among 20 sizes only 1 x 100,000 x 64, 10.9 (10.6).
int conv_strip(int B, int T, int by, int ny, int cta_bytes, int per_sm, int n_sm) {
    int best = kConvBatch;
    float least = 0.f;
    for (int strip = kConvBatch; strip <= kConvStrip; strip += strip < 64 ? kConvBatch : 2 * kConvBatch) {
        const long long ctas = ((long long)B * ((T - 1) / strip + 1) + by - 1) / by * ny, n = (ctas + n_sm - 1) / n_sm;
        const float walk = static_cast<float>(strip < T ? strip : T);
        auto round = [&](long long held) { return 13.f + walk * std::max(1.f, held * cta_bytes / 57.f); };
        const float t = n / per_sm * round(per_sm) + (n % per_sm ? round(n % per_sm) : 0.f);
        if (strip == kConvBatch || t < least) least = t, best = strip;
        if (strip >= T) break;
    }
    return best;
}

template <typename E, int VEC, int W> cudaError_t conv_run(ConvParams &p, bool step, int n_sm, cudaStream_t stream) {
    const int nv = (p.E + VEC - 1) / VEC;
    const int ny = (nv + kConvThreads - 1) / kConvThreads;
    const int bx = (nv + ny - 1) / ny, by = kConvThreads / bx;  // bx <= 256
    p.strip = p.strips = 1;
    if (!step) {
        int per_sm = 0;
        const cudaError_t e = conv_fit<E, VEC, W>(bx * by, &per_sm);
        if (e != cudaSuccess) return e;
        const int raw = static_cast<int>(sizeof(typename Vec<E, VEC>::raw));
        p.strip = conv_strip(p.B, p.grid.T, by, ny, (bx * by + 31) / 32 * (raw < 4 ? 4 : raw), per_sm, n_sm);
        p.strips = (p.grid.T - 1) / p.strip + 1;
    }
    p.items = (long long)p.B * p.strips;
    const long long rows = step ? p.B : p.items, gx = (rows + by - 1) / by;
    if (gx > 0x7fffffffLL || ny > 65535) return cudaErrorInvalidValue;
    const dim3 grid(static_cast<unsigned>(gx), ny), block(bx, by);
    if (step)
        conv_step_kernel<E, VEC, W><<<grid, block, 0, stream>>>(p);
    else
        conv_kernel<E, VEC, W><<<grid, block, conv_smem_bytes<E, VEC>(bx * by), stream>>>(p);
    return cudaGetLastError();
}
template <typename E, int VEC> cudaError_t conv_run_w(ConvParams &p, int W, bool step, int n_sm, cudaStream_t s) {
    if (W == 2) return conv_run<E, VEC, 2>(p, step, n_sm, s);
    if (W == 3) return conv_run<E, VEC, 3>(p, step, n_sm, s);
    return conv_run<E, VEC, 4>(p, step, n_sm, s);
}
// Four channels a thread, two (16-bit elements) or one: what every row starts and ends on.  (Eight fp16 channels'
// window, taps and loads do not fit the registers of 512 threads an SM.)
template <typename E> cudaError_t conv_run_e(ConvParams &p, int W, bool step, int n_sm, cudaStream_t s) {
    if (p.E % 4 == 0 && p.x_stride % 4 == 0) return conv_run_w<E, 4>(p, W, step, n_sm, s);
    if constexpr (sizeof(E) == 2) {
        if (p.E % 2 == 0 && p.x_stride % 2 == 0) return conv_run_w<E, 2>(p, W, step, n_sm, s);
    }
    return conv_run_w<E, 1>(p, W, step, n_sm, s);
}

}  // namespace

cudaError_t launch_conv(const ConvProblem &q, bool step, cudaStream_t stream) {
    ConvParams p;
    p.x = q.x;
    p.x_stride = q.x_stride;
    p.w = q.weight;
    p.b = q.bias;
    p.init = q.state_in;
    p.out = q.out;
    p.state = q.state_out;
    p.grid = make_scan_grid(q.grid_h, q.grid_w, q.order);
    p.B = q.B;
    p.E = q.E;
    p.silu = q.silu;
    int n_sm = 0;
    const cudaError_t e = sm_count(&n_sm);
    if (e != cudaSuccess) return e;
    if (q.dtype == 0) return conv_run_e<float>(p, q.W, step, n_sm, stream);
    if (q.dtype == 1) return conv_run_e<__half>(p, q.W, step, n_sm, stream);
    return conv_run_e<__nv_bfloat16>(p, q.W, step, n_sm, stream);
}

}  // namespace gtr
