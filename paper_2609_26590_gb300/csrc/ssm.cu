// ssm.cu -- selective state-space scan along a scan order, for whole sequences and single tokens:
//   dt = softplus(delta + bias),  h_s[n] = exp(dt A[n]) h_{s-1}[n] + dt x_s B_s[n],
//   y_s = (sum_n C_s[n] h_s[n] + D x_s) SiLU(z_s)
// per channel, with N states a channel, A and D of the channel and B_s, C_s of the token.
//
// A decay of its own for every (channel, state) leaves nothing for the tensor cores: the work is one
// power of two and four multiply-adds a token, channel and state on the CUDA cores.  LPC lanes share a
// channel's states, NS each in packed fp32 pairs; a warp owns 32 / LPC channels and walks the
// positions of its segment in blocks of 16: the lanes stage dt, dt x, B and C as fp32 in the warp's
// shared memory (no barrier beyond the warp), then every lane steps its states.  The LPC partial
// readouts of LPC tokens are exchanged at once so that each lane ends with the whole readout of the
// token it loaded x and z of, and stores it.
//
// Few channels leave SMs idle, so short launches cut the sequence into one segment a warp of the
// CTA: a first walk yields each segment's end state from zero and its sum of dt (the segment's
// decay is exp(A sum dt)), the CTA folds them in order, and the second walk starts from the fold.
#include <cuda_runtime.h>

#include "elem.cuh"
#include "f32x2.cuh"
#include "gla_internal.h"
#include "scanpos.cuh"

namespace gtr {
namespace {

constexpr int kSsmBlock = 16;     // positions staged at once
constexpr int kSsmMaxWarps = 16;  // segments of a CTA
constexpr int kSsmWarps = 4;      // channel groups of a CTA that does not split
constexpr float kLog2e = 1.4426950408889634f;

struct SsmParams {
    const void *x, *delta, *z, *Bm, *C;
    long long x_stride, delta_stride, z_stride, b_stride, c_stride;
    const float *A, *D, *bias, *init;
    void *out;
    float *state;
    ScanGrid grid;
    int B, E, N, softplus;
    int groups;   // channel groups of a sequence
    int nseg, seg_len;
};

__device__ __forceinline__ float exp2_hw(float a) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(a));
    return r;
}

// softplus(v) = max(v, 0) + log(1 + e^{-|v|}): log1p keeps the small steps of very negative v.
__device__ __forceinline__ float softplus(float v) { return fmaxf(v, 0.f) + log1pf(__expf(-fabsf(v))); }

// Sum over the LPC lanes of a channel of LPC values each: lane q ends with the sum of value q.
template <int LPC> __device__ __forceinline__ float exchange_sum(float (&v)[LPC], int q) {
#pragma unroll
    for (int o = LPC / 2; o > 0; o >>= 1) {
        const bool hi = q & o;
#pragma unroll
        for (int i = 0; i < o; ++i) {
            const float keep = hi ? v[i + o] : v[i], send = hi ? v[i] : v[i + o];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
        }
    }
    return v[0];
}

template <typename E, int LPC, int NS>
__global__ void __launch_bounds__(kSsmMaxWarps * 32) ssm_kernel(const __grid_constant__ SsmParams p) {
    constexpr int CH = 32 / LPC, NP = LPC * NS, TL = kSsmBlock / LPC, NB = kSsmBlock * NP / 32;
    constexpr int kWarpFloats = kSsmBlock * (2 * CH + 2 * NP);
    extern __shared__ float4 smem4[];
    float *smem = reinterpret_cast<float *>(smem4);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, ch = lane / LPC, q = lane % LPC;
    const bool split = p.nseg > 1;
    const long long unit = split ? blockIdx.x : (long long)blockIdx.x * kSsmWarps + warp;
    if (unit >= (long long)p.B * p.groups) return;  // whole warps, and only where the CTA has no barrier
    const int b = static_cast<int>(unit / p.groups), c = static_cast<int>(unit - (long long)b * p.groups) * CH + ch;
    const bool live = c < p.E;
    const int T = p.grid.T;
    const int seg = split ? warp : 0;
    const int t0 = split ? (seg * p.seg_len < T ? seg * p.seg_len : T) : 0;
    const int t1 = split ? (T - t0 < p.seg_len ? T : t0 + p.seg_len) : T;
    float2 *s_dt = reinterpret_cast<float2 *>(smem + (size_t)warp * kWarpFloats);  // [block][CH]: dt, dt x
    float *s_b = smem + (size_t)warp * kWarpFloats + 2 * kSsmBlock * CH;            // [block][NP]
    float *s_c = s_b + kSsmBlock * NP;
    const long long seq = (long long)b * T;
    const E *x = static_cast<const E *>(p.x) + seq * p.x_stride + (live ? c : 0);
    const E *dl = static_cast<const E *>(p.delta) + seq * p.delta_stride + (live ? c : 0);
    const E *z = p.z ? static_cast<const E *>(p.z) + seq * p.z_stride + (live ? c : 0) : nullptr;
    const E *Bm = static_cast<const E *>(p.Bm) + seq * p.b_stride;
    const E *C = static_cast<const E *>(p.C) + seq * p.c_stride;
    E *out = static_cast<E *>(p.out) + seq * p.E + (live ? c : 0);
    const float bias = p.bias && live ? p.bias[c] : 0.f, skip = p.D && live ? p.D[c] : 0.f;
    f2 a2[NS / 2], h[NS / 2];
#pragma unroll
    for (int i = 0; i < NS / 2; ++i) {
        float v[2], s[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int n = q * NS + 2 * i + k;
            const bool in = live && n < p.N;
            v[k] = in ? p.A[(long long)c * p.N + n] * kLog2e : 0.f;
            s[k] = in && p.init ? p.init[((long long)b * p.E + c) * p.N + n] : 0.f;
        }
        a2[i] = pack2(v[0], v[1]);
        h[i] = pack2(s[0], s[1]);
    }
    float sum_dt = 0.f;

    auto walk = [&](bool readout) {
        for (int s0 = t0; s0 < t1; s0 += kSsmBlock) {
            float xv[TL], zv[TL];
            int tok[TL];
            __syncwarp();
#pragma unroll
            for (int j = 0; j < TL; ++j) {
                const int s = s0 + j * LPC + q;
                const bool in = live && s < t1;
                ScanPos pos;
                pos.set(p.grid, in ? s : t0);
                tok[j] = pos.t;
                float dt = 0.f;
                xv[j] = zv[j] = 0.f;
                if (in) {
                    xv[j] = to_f32(x[pos.t * p.x_stride]);
                    dt = to_f32(dl[pos.t * p.delta_stride]) + bias;
                    if (p.softplus) dt = softplus(dt);
                    if (readout && z) zv[j] = to_f32(z[pos.t * p.z_stride]);
                }
                s_dt[(j * LPC + q) * CH + ch] = make_float2(dt, dt * xv[j]);
            }
#pragma unroll
            for (int k = 0; k < NB; ++k) {
                const int i = k * 32 + lane, s = s0 + i / NP, n = i % NP;
                float vb = 0.f, vc = 0.f;
                if (s < t1 && n < p.N) {
                    ScanPos pos;
                    pos.set(p.grid, s);
                    vb = to_f32(Bm[pos.t * p.b_stride + n]);
                    if (readout) vc = to_f32(C[pos.t * p.c_stride + n]);
                }
                s_b[i] = vb;
                s_c[i] = vc;
            }
            __syncwarp();
#pragma unroll
            for (int j = 0; j < TL; ++j) {
                float part[LPC];
#pragma unroll
                for (int u = 0; u < LPC; ++u) {
                    const int t = j * LPC + u;
                    const float2 d = s_dt[t * CH + ch];
                    const f2 dt2 = pack2(d.x, d.x), du2 = pack2(d.y, d.y);
                    const f2 *bp = reinterpret_cast<const f2 *>(s_b + t * NP + q * NS);
                    const f2 *cp = reinterpret_cast<const f2 *>(s_c + t * NP + q * NS);
                    f2 acc = 0;
                    sum_dt += d.x;
#pragma unroll
                    for (int i = 0; i < NS / 2; ++i) {
                        const float2 e = unpack2(mul2(dt2, a2[i]));
                        h[i] = fma2(pack2(exp2_hw(e.x), exp2_hw(e.y)), h[i], mul2(du2, bp[i]));
                        acc = fma2(cp[i], h[i], acc);
                    }
                    const float2 r = unpack2(acc);
                    part[u] = r.x + r.y;
                }
                if (readout) {
                    float y = exchange_sum<LPC>(part, q);
                    y = fmaf(skip, xv[j], y);
                    if (z) y *= silu<E>(zv[j]);
                    if (live && s0 + j * LPC + q < t1) out[(long long)tok[j] * p.E] = from_f32<E>(y);
                }
            }
        }
    };

    if (split) {
        float *sum_h = smem + (size_t)p.nseg * kWarpFloats;  // [nseg][CH][NP]
        float *sum_d = sum_h + (size_t)p.nseg * CH * NP;     // [nseg][CH]
        f2 start[NS / 2];
#pragma unroll
        for (int i = 0; i < NS / 2; ++i) start[i] = h[i], h[i] = 0;
        if (seg + 1 < p.nseg) {  // nothing follows the last segment
            walk(false);
#pragma unroll
            for (int i = 0; i < NS / 2; ++i)
                reinterpret_cast<f2 *>(sum_h + ((size_t)seg * CH + ch) * NP + q * NS)[i] = h[i];
            if (q == 0) sum_d[seg * CH + ch] = sum_dt;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NS / 2; ++i) h[i] = start[i];
        for (int j = 0; j < seg; ++j) {
            const float d = sum_d[j * CH + ch];
            const f2 *e = reinterpret_cast<const f2 *>(sum_h + ((size_t)j * CH + ch) * NP + q * NS);
#pragma unroll
            for (int i = 0; i < NS / 2; ++i) {
                const float2 m = unpack2(mul2(pack2(d, d), a2[i]));
                h[i] = fma2(pack2(exp2_hw(m.x), exp2_hw(m.y)), h[i], e[i]);
            }
        }
    }
    walk(true);
    if (p.state && live && seg + 1 == p.nseg) {
#pragma unroll
        for (int i = 0; i < NS / 2; ++i) {
            const float2 v = unpack2(h[i]);
            float *dst = p.state + ((long long)b * p.E + c) * p.N;
            const int n = q * NS + 2 * i;
            if (n < p.N) dst[n] = v.x;
            if (n + 1 < p.N) dst[n + 1] = v.y;
        }
    }
}

// One token of every sequence.  Memory-bound: the states are read and written once.  Four states a
// thread in one 16-byte access, N / 4 neighbouring lanes a channel (N / 4 a power of two).
template <typename E, int LPC>
__global__ void __launch_bounds__(256) ssm_step_kernel(const __grid_constant__ SsmParams p) {
    const int per = p.E * LPC;  // threads a sequence
    const int blocks = (per + 255) / 256;
    const int b = blockIdx.x / blocks, i = (blockIdx.x - b * blocks) * 256 + threadIdx.x;
    const bool live = i < per;
    const int c = live ? i / LPC : 0, q = i % LPC;
    const float u = to_f32(static_cast<const E *>(p.x)[(long long)b * p.x_stride + c]);
    float dt = to_f32(static_cast<const E *>(p.delta)[(long long)b * p.delta_stride + c]) + (p.bias ? p.bias[c] : 0.f);
    if (p.softplus) dt = softplus(dt);
    const long long at = ((long long)b * p.E + c) * (4 * LPC) + 4 * q;
    const float4 a = *reinterpret_cast<const float4 *>(p.A + (long long)c * (4 * LPC) + 4 * q);
    const float4 h = *reinterpret_cast<const float4 *>(p.init + at);
    const E *Bm = static_cast<const E *>(p.Bm) + (long long)b * p.b_stride + 4 * q;
    const E *C = static_cast<const E *>(p.C) + (long long)b * p.c_stride + 4 * q;
    const float du = dt * u, av[4] = {a.x, a.y, a.z, a.w}, hv[4] = {h.x, h.y, h.z, h.w};
    float n[4], y = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        n[k] = fmaf(exp2_hw(dt * (av[k] * kLog2e)), hv[k], du * to_f32(Bm[k]));
        y = fmaf(to_f32(C[k]), n[k], y);
    }
    if (live) *reinterpret_cast<float4 *>(p.state + at) = make_float4(n[0], n[1], n[2], n[3]);
#pragma unroll
    for (int o = LPC / 2; o > 0; o >>= 1) y += __shfl_xor_sync(0xffffffffu, y, o);
    if (live && q == 0) {
        if (p.D) y = fmaf(p.D[c], u, y);
        if (p.z) y *= silu<E>(to_f32(static_cast<const E *>(p.z)[(long long)b * p.z_stride + c]));
        static_cast<E *>(p.out)[(long long)b * p.E + c] = from_f32<E>(y);
    }
}

// The same for any number of states: a thread a channel.
template <typename E> __global__ void __launch_bounds__(128) ssm_step_any_kernel(const __grid_constant__ SsmParams p) {
    const int blocks = (p.E + 127) / 128;
    const int b = blockIdx.x / blocks, c = (blockIdx.x - b * blocks) * 128 + threadIdx.x;
    if (c >= p.E) return;
    const float u = to_f32(static_cast<const E *>(p.x)[(long long)b * p.x_stride + c]);
    float dt = to_f32(static_cast<const E *>(p.delta)[(long long)b * p.delta_stride + c]) + (p.bias ? p.bias[c] : 0.f);
    if (p.softplus) dt = softplus(dt);
    const long long at = ((long long)b * p.E + c) * p.N;
    const E *Bm = static_cast<const E *>(p.Bm) + (long long)b * p.b_stride;
    const E *C = static_cast<const E *>(p.C) + (long long)b * p.c_stride;
    const float du = dt * u;
    float y = 0.f;
    for (int n = 0; n < p.N; ++n) {
        const float h = fmaf(exp2_hw(dt * (p.A[(long long)c * p.N + n] * kLog2e)), p.init[at + n], du * to_f32(Bm[n]));
        p.state[at + n] = h;
        y = fmaf(to_f32(C[n]), h, y);
    }
    if (p.D) y = fmaf(p.D[c], u, y);
    if (p.z) y *= silu<E>(to_f32(static_cast<const E *>(p.z)[(long long)b * p.z_stride + c]));
    static_cast<E *>(p.out)[(long long)b * p.E + c] = from_f32<E>(y);
}

SsmParams ssm_params(const SsmProblem &q) {
    SsmParams p;
    p.x = q.x, p.delta = q.delta, p.z = q.z, p.Bm = q.Bm, p.C = q.C;
    p.x_stride = q.x_stride, p.delta_stride = q.delta_stride, p.z_stride = q.z_stride;
    p.b_stride = q.b_stride, p.c_stride = q.c_stride;
    p.A = q.A, p.D = q.D, p.bias = q.delta_bias, p.init = q.state_in;
    p.out = q.out, p.state = q.state_out;
    p.grid = make_scan_grid(q.grid_h, q.grid_w, q.order);
    p.B = q.B, p.E = q.E, p.N = q.N, p.softplus = q.softplus;
    p.groups = p.nseg = p.seg_len = 0;
    return p;
}

template <typename E, int LPC, int NS> cudaError_t ssm_run(SsmParams &p, int n_sm, cudaStream_t stream) {
    constexpr int CH = 32 / LPC, NP = LPC * NS;
    constexpr int kWarpFloats = kSsmBlock * (2 * CH + 2 * NP);
    p.groups = (p.E + CH - 1) / CH;
    const long long units = (long long)p.B * p.groups;
    // split while the warps would not fill the SMs' schedulers twice, at least two blocks a segment
    const int blocks = (p.grid.T - 1) / kSsmBlock + 1;
    int cap = kSsmMaxWarps;
    while ((size_t)cap * (kWarpFloats + CH * NP + CH) * sizeof(float) > 48 * 1024) cap /= 2;
    long long want = 8LL * n_sm / units;
    if (want > cap) want = cap;
    if (want > blocks / 2) want = blocks / 2;
    p.nseg = want < 2 ? 1 : static_cast<int>(want);
    const int per = (blocks + p.nseg - 1) / p.nseg;
    p.nseg = (blocks + per - 1) / per;  // no empty segment
    p.seg_len = per * kSsmBlock;
    const int warps = p.nseg > 1 ? p.nseg : kSsmWarps;
    const long long ctas = p.nseg > 1 ? units : (units + kSsmWarps - 1) / kSsmWarps;
    if (ctas > 0x7fffffffLL) return cudaErrorInvalidValue;
    const size_t smem = (size_t)warps * (kWarpFloats + (p.nseg > 1 ? CH * NP + CH : 0)) * sizeof(float);
    ssm_kernel<E, LPC, NS><<<static_cast<unsigned>(ctas), warps * 32, smem, stream>>>(p);
    return cudaGetLastError();
}
template <typename E> cudaError_t ssm_run_n(SsmParams &p, int n_sm, cudaStream_t s) {
    if (p.N <= 8) return ssm_run<E, 2, 4>(p, n_sm, s);
    if (p.N <= 16) return ssm_run<E, 4, 4>(p, n_sm, s);
    if (p.N <= 32) return ssm_run<E, 8, 4>(p, n_sm, s);
    return ssm_run<E, 8, 8>(p, n_sm, s);
}

template <typename E> cudaError_t ssm_step_e(SsmParams &p, cudaStream_t s) {
    const int lpc = p.N % 4 == 0 ? p.N / 4 : 0;
    const long long per = lpc && !(lpc & (lpc - 1)) ? ((long long)p.E * lpc + 255) / 256 : ((long long)p.E + 127) / 128;
    if (per * p.B > 0x7fffffffLL) return cudaErrorInvalidValue;
    const unsigned ctas = static_cast<unsigned>(per * p.B);
    switch (lpc) {
    case 1: ssm_step_kernel<E, 1><<<ctas, 256, 0, s>>>(p); break;
    case 2: ssm_step_kernel<E, 2><<<ctas, 256, 0, s>>>(p); break;
    case 4: ssm_step_kernel<E, 4><<<ctas, 256, 0, s>>>(p); break;
    case 8: ssm_step_kernel<E, 8><<<ctas, 256, 0, s>>>(p); break;
    case 16: ssm_step_kernel<E, 16><<<ctas, 256, 0, s>>>(p); break;
    default: ssm_step_any_kernel<E><<<ctas, 128, 0, s>>>(p);
    }
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_ssm(const SsmProblem &q, cudaStream_t stream) {
    int n_sm = 0;
    const cudaError_t e = sm_count(&n_sm);
    if (e != cudaSuccess) return e;
    SsmParams p = ssm_params(q);
    if (q.dtype == 0) return ssm_run_n<float>(p, n_sm, stream);
    if (q.dtype == 1) return ssm_run_n<__half>(p, n_sm, stream);
    return ssm_run_n<__nv_bfloat16>(p, n_sm, stream);
}

cudaError_t launch_ssm_step(const SsmProblem &q, cudaStream_t stream) {
    SsmParams p = ssm_params(q);
    if (q.dtype == 0) return ssm_step_e<float>(p, stream);
    if (q.dtype == 1) return ssm_step_e<__half>(p, stream);
    return ssm_step_e<__nv_bfloat16>(p, stream);
}

}  // namespace gtr
