// ffn.cu -- the gated feed-forward step and its backward pass on the tensor cores:
//   G = X Wg^T, V = X Wv^T, H = SiLU(G) V                       X [M, D], Wg and Wv [F, D], H [M, F]
//   dV = dH SiLU(G), dG = dH V s(G) (1 + G (1 - s(G)))          s: the logistic function
//   dX = dG Wg + dV Wv,  dWg = dG^T X,  dWv = dV^T X
//
// Four products of one persistent kernel, which differ in their operands' major-ness and in what
// happens to the fp32 accumulator on its way out:
//   kFwd  both projections of 128 channels as one 256-column tile (gate columns from the even CTA's
//         weights, value columns from the odd one's), SiLU and the product in registers, H stored
//   kAct  the same projections again (nothing of M x F is kept between the passes), dH read beside
//         them, dG and dV stored in the inputs' type: they are operands of the next two products,
//         which the tensor cores take in 16 bits (half a step of rounding each)
//   kDx   [dG dV] [Wg; Wv], the weights read along F (MN-major)
//   kDw   dG^T X and dV^T X, both operands read along the tokens (MN-major)
//
// A CTA pair (tcgen05 cta_group::2) computes 256 x 256 (128) tiles: 64-deep blocks of both operands
// arrive by TMA in 128-byte-swizzled shared memory (rows and columns outside the tensors as zeros),
// one warp issues the MMAs, and eight warps empty one TMEM accumulator while the next tile fills
// the other.  Every wait is bounded; a kernel that gives up sets the status word.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <atomic>
#include <cstdint>
#include <cstring>

#include "elem.cuh"
#include "f32x2.cuh"
#include "fastdiv.cuh"
#include "gla_internal.h"
#include "tc_ptx.cuh"

namespace gtr {

__device__ unsigned int g_ffn_status;

namespace {

using namespace ptx;

enum : int { kFwd = 0, kAct = 1, kDx = 2, kDw = 3 };

constexpr int kFfnThreads = 384;   // warps: loads, MMAs, TMEM, idle, eight epilogue warps
constexpr int kFfnEpiWarp = 4;
constexpr int kTileM = 256;        // accumulator rows of a CTA pair
constexpr int kBlockK = 64;        // 128 bytes of an operand row
constexpr int kStageA = 128 * 128; // bytes of a CTA's half of A, and of B
constexpr int kStageBytes = 2 * kStageA;
constexpr int kBox = 32 * 128;     // an epilogue warp's box: 32 rows x 64 columns of 16 bits
constexpr uint64_t kFfnWaitNs = 1000000000ull;

constexpr int ffn_stages(int mode) { return mode == kAct ? 5 : 6; }
constexpr int ffn_boxes(int mode) { return mode == kAct ? 2 : 1; }  // staging boxes of a warp
constexpr size_t ffn_smem(int mode) {
    return (size_t)ffn_stages(mode) * kStageBytes + 8 * (size_t)ffn_boxes(mode) * kBox + 1024;
}

struct FfnParams {
    CUtensorMap a[2], b[2];  // operands (the second: the odd CTA's weights, or the second half of the product)
    CUtensorMap o[2];        // outputs
    CUtensorMap dh;          // kAct
    FastDiv tm;              // tiles down the rows
    int tiles;
    int nk, nk_half;         // 64-deep blocks of a tile; of one of kDx's two products
    int rows, cols;          // extent of an output
    int bn;                  // columns of a tile's accumulator
    uint32_t idesc;
};

struct FfnBars {
    uint64_t full[6], empty[6], acc_full[2], acc_empty[2], dh[8];
    uint32_t tmem, abort;
};

// The logistic function of a pair by the hardware's 2^x and 1/x (a few 2^-22).  Flushing their subnormal results
// changes nothing: 1 + e is 1 there, and 1 / (1 + e) is below 2^-126.
__device__ __forceinline__ f2 sigmoid2(f2 z) {
    const float kNegLog2e = -1.4426950408889634f;
    const float2 t = unpack2(mul2(z, pack2(kNegLog2e, kNegLog2e)));
    float e0, e1, r0, r1;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(t.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(t.y));
    const float2 d = unpack2(add2(pack2(e0, e1), pack2(1.f, 1.f)));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(d.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(d.y));
    return pack2(r0, r1);
}

template <int MODE, typename E>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kFfnThreads, 1) ffn_kernel(const __grid_constant__ FfnParams p) {
    constexpr bool A_MN = MODE == kDw, B_MN = MODE == kDx || MODE == kDw;
    constexpr int S = ffn_stages(MODE), BOXES = ffn_boxes(MODE);
    extern __shared__ uint8_t ffn_raw[];
    __shared__ FfnBars bars;
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(ffn_raw) + 1023) & ~uintptr_t(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    volatile uint32_t *abort = &bars.abort;

    if (threadIdx.x == 0) {
        for (int i = 0; i < S; ++i) mbar_init(&bars.full[i], 1), mbar_init(&bars.empty[i], 1);
        for (int i = 0; i < 2; ++i) mbar_init(&bars.acc_full[i], 1), mbar_init(&bars.acc_empty[i], 16);
        for (int i = 0; i < 8; ++i) mbar_init(&bars.dh[i], 1);
        bars.abort = 0;
        fence_mbar_init();
    }
    if (warp == 2) {
        tmem_alloc_pair(&bars.tmem, 512);
        tmem_relinquish_pair();
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    __syncwarp();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = bars.tmem;

    auto give_up = [&] {
        *abort = 1;
        atomicOr(&g_ffn_status, kStatusTimeout);
    };

    if (warp == 0) {
        if (lane == 0) {
            // ---- loads: this CTA's half of A's rows and of B's columns, counted on the even CTA's barrier
            const int bhalf = p.bn / 2;
            const uint32_t bytes = 2u * (kStageA + static_cast<uint32_t>(bhalf) * 128u);
            uint32_t it = 0;
            bool ok = true;
            for (int tile = pair; ok && tile < p.tiles; tile += pairs) {
                const int n = fdiv(tile, p.tm), m = tile - n * p.tm.d;
                for (int k = 0; k < p.nk; ++k, ++it) {
                    const uint32_t s = it % S;
                    if (it >= S && !mbar_wait(&bars.empty[s], ((it / S) - 1) & 1, abort, kFfnWaitNs)) {
                        give_up();
                        ok = false;
                        break;
                    }
                    const uint32_t bar = map_to_cta(smem_u32(&bars.full[s]), 0);
                    if (rank == 0) mbar_arrive_expect_tx(&bars.full[s], bytes);
                    const uint32_t sa = smem_u32(smem) + s * kStageBytes, sb = sa + kStageA;
                    if constexpr (MODE == kFwd || MODE == kAct) {
                        tma_load_2d_pair(sa, &p.a[0], bar, k * kBlockK, m * kTileM + rank * 128);
                        tma_load_2d_pair(sb, &p.b[rank], bar, k * kBlockK, n * 128);
                    } else if constexpr (MODE == kDx) {
                        const int half = k >= p.nk_half, kk = (k - half * p.nk_half) * kBlockK;
                        tma_load_2d_pair(sa, &p.a[half], bar, kk, m * kTileM + rank * 128);
                        for (int j = 0; j < bhalf; j += 64)
                            tma_load_2d_pair(sb + j * 128, &p.b[half], bar, n * p.bn + rank * bhalf + j, kk);
                    } else {
                        const int mt = p.tm.d / 2, g = m >= mt, m0 = (m - g * mt) * kTileM + rank * 128;
                        for (int j = 0; j < 128; j += 64)
                            tma_load_2d_pair(sa + j * 128, &p.a[g], bar, m0 + j, k * kBlockK);
                        for (int j = 0; j < bhalf; j += 64)
                            tma_load_2d_pair(sb + j * 128, &p.b[0], bar, n * p.bn + rank * bhalf + j, k * kBlockK);
                    }
                }
            }
            // every block consumed: no copy and no barrier arrival is in flight any more
            const uint32_t last = it < S ? it : S;
            for (uint32_t i = it - last; i != it; ++i)
                if (!mbar_wait(&bars.empty[i % S], (i / S) & 1, nullptr, kFfnWaitNs)) give_up();
        }
    } else if (warp == 1) {
        if (rank == 0) {
            // ---- MMAs of both CTAs' halves
            uint32_t it = 0, acc = 0;
            bool ok = true;
            for (int tile = pair; ok && tile < p.tiles; tile += pairs, ++acc) {
                const uint32_t buf = acc & 1;
                if (acc >= 2) ok = mbar_wait_cluster(&bars.acc_empty[buf], ((acc >> 1) - 1) & 1, abort, kFfnWaitNs);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                for (int k = 0; k < p.nk; ++k, ++it) {
                    const uint32_t s = it % S;
                    ok = __all_sync(0xffffffffu, mbar_wait_cluster(&bars.full[s], (it / S) & 1, abort, kFfnWaitNs));
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t sa = smem_u32(smem) + s * kStageBytes, sb = sa + kStageA;
                    const uint64_t ad = smem_desc(sa, A_MN ? 8192 : 16, 1024, kLayoutSw128);
                    const uint64_t bd = smem_desc(sb, B_MN ? 8192 : 16, 1024, kLayoutSw128);
                    mma4_f16_ss_pair<A_MN ? 128 : 2, B_MN ? 128 : 2>(tmem + buf * 256, ad, bd, p.idesc, k > 0);
                    mma_commit_pair(&bars.empty[s]);
                }
                if (ok) mma_commit_pair(&bars.acc_full[buf]);
            }
            if (!ok && lane == 0) give_up();
        }
    } else if (warp >= kFfnEpiWarp) {
        // ---- epilogue: rows 32 (warp % 4) .. of this CTA's 128, one half of the columns
        const int w = warp - kFfnEpiWarp, sub = warp & 3, half = w >> 2;
        uint8_t *box = smem + S * kStageBytes + (size_t)w * BOXES * kBox;
        const uint32_t lanes = static_cast<uint32_t>(sub * 32) << 16;
        const uint32_t acc_empty = map_to_cta(smem_u32(&bars.acc_empty[0]), 0);  // the even CTA's, 8 bytes apart
        uint32_t acc = 0;
        for (int tile = pair; tile < p.tiles; tile += pairs, ++acc) {
            const int n = fdiv(tile, p.tm), m = tile - n * p.tm.d;
            const uint32_t buf = acc & 1;
            int row0 = m * kTileM + static_cast<int>(rank) * 128 + sub * 32, group = 0;
            if constexpr (MODE == kDw) {
                const int mt = p.tm.d / 2;
                group = m >= mt;
                row0 -= group * mt * kTileM;
            }
            if constexpr (MODE == kAct) {
                if (lane == 0) {
                    bulk_wait_read();  // the box of the tile before has been stored
                    mbar_arrive_expect_tx(&bars.dh[w], kBox);
                    tma_load_2d(box, &p.dh, &bars.dh[w], n * 128 + half * 64, row0);
                }
            }
            bool ok = mbar_wait(&bars.acc_full[buf], (acc >> 1) & 1, abort, kFfnWaitNs);
            if constexpr (MODE == kAct) ok = mbar_wait(&bars.dh[w], acc & 1, nullptr, kFfnWaitNs) && ok;
            if (!__all_sync(0xffffffffu, ok)) {
                if (lane == 0) give_up();
                break;
            }
            tc_fence_after();
            const uint32_t taddr = tmem + buf * 256 + lanes;
            if constexpr (MODE == kFwd || MODE == kAct) {
                if (MODE == kFwd) {
                    if (lane == 0) bulk_wait_read();
                    __syncwarp();
                }
                const int col0 = n * 128 + half * 64;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t g[32], v[32];
                    tmem_ld_32x32(taddr + half * 64 + c * 32, g);
                    tmem_ld_32x32(taddr + 128 + half * 64 + c * 32, v);
                    tmem_ld_wait();
                    if (c == 1) {  // the accumulator is in registers
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster_relaxed(acc_empty + 8 * buf);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {  // 16 bytes: eight columns
                        uint4 *at = reinterpret_cast<uint4 *>(box + lane * 128 + (((c * 4 + j) ^ (lane & 7)) << 4));
                        uint32_t in[4], o0[4], o1[4];
                        if constexpr (MODE == kAct) {
                            const uint4 d = *at;
                            in[0] = d.x, in[1] = d.y, in[2] = d.z, in[3] = d.w;
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const f2 z = pack2(g[8 * j + 2 * i], g[8 * j + 2 * i + 1]);
                            const f2 y = pack2(v[8 * j + 2 * i], v[8 * j + 2 * i + 1]), sg = sigmoid2(z);
                            if constexpr (MODE == kFwd) {
                                const float2 h = unpack2(mul2(mul2(z, sg), y));
                                o0[i] = pack16<E>(h.x, h.y);
                            } else {
                                const float2 d = unpack16<E>(in[i]);
                                const f2 one = pack2(1.f, 1.f), ds = mul2(pack2(d.x, d.y), sg);
                                // dG = dH V s (1 + G (1 - s)), dV = dH s G
                                const float2 dg = unpack2(mul2(mul2(ds, y), fma2(z, fma2(sg, pack2(-1.f, -1.f), one), one)));
                                const float2 dv = unpack2(mul2(ds, z));
                                o0[i] = pack16<E>(dg.x, dg.y);
                                o1[i] = pack16<E>(dv.x, dv.y);
                            }
                        }
                        *at = make_uint4(o0[0], o0[1], o0[2], o0[3]);
                        if constexpr (MODE == kAct)
                            *reinterpret_cast<uint4 *>(reinterpret_cast<uint8_t *>(at) + kBox) = make_uint4(o1[0], o1[1], o1[2], o1[3]);
                    }
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0 && row0 < p.rows && col0 < p.cols) {
                    tma_store_2d(&p.o[0], box, col0, row0);
                    if constexpr (MODE == kAct) tma_store_2d(&p.o[1], box + kBox, col0, row0);
                    bulk_commit();
                }
            } else {
                const int width = p.bn / 2;
                for (int b0 = 0; b0 < width; b0 += 64) {
                    const int off = half * width + b0, col0 = n * p.bn + off;
                    if (lane == 0) bulk_wait_read();
                    __syncwarp();
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t g[32];
                        tmem_ld_32x32(taddr + off + c * 32, g);
                        tmem_ld_wait();
                        if (c == 1 && b0 + 64 >= width) {
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive_cluster_relaxed(acc_empty + 8 * buf);
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float o0[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) o0[i] = __uint_as_float(g[8 * j + i]);
                            *reinterpret_cast<uint4 *>(box + lane * 128 + (((c * 4 + j) ^ (lane & 7)) << 4)) =
                                Vec<E, 8>::pack(o0);
                        }
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0 && row0 < p.rows && col0 < p.cols) {
                        tma_store_2d(&p.o[group], box, col0, row0);
                        bulk_commit();
                    }
                }
            }
        }
        if (lane == 0) bulk_wait_all();
    }
    __syncwarp();  // the barriers below are the whole warp's
    tc_fence_before();
    __syncthreads();
    __syncwarp();
    cluster_sync();  // neither CTA leaves while the other may still signal it or use its TMEM
    tc_fence_after();
    if (warp == 2) tmem_dealloc_pair(tmem, 512);
}

// A row-major matrix [rows][cols] of 16-bit elements at `stride` elements a row, in boxes of 64 columns
// (128 swizzled bytes) x box_rows.
bool ffn_map(CUtensorMap *m, const void *base, int dtype, long long rows, long long cols, long long stride, int box_rows) {
    auto enc = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(tensor_map_encoder());
    if (!enc) return false;
    cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
    cuuint64_t strides[1] = {static_cast<cuuint64_t>(stride) * 2};
    cuuint32_t box[2] = {64, static_cast<cuuint32_t>(box_rows)}, estr[2] = {1, 1};
    return enc(m, dtype == 1 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2,
               const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int MODE, typename E> cudaError_t ffn_launch_typed(const FfnParams &p, int n_sm, cudaStream_t stream) {
    static std::atomic<unsigned long long> set_on_devices(0);
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = 1ull << (dev & 63);
    if (!(set_on_devices.load(std::memory_order_relaxed) & bit)) {
        e = cudaFuncSetAttribute(ffn_kernel<MODE, E>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 static_cast<int>(ffn_smem(MODE)));
        if (e != cudaSuccess) return e;
        set_on_devices.fetch_or(bit);
    }
    const int pairs = p.tiles < n_sm / 2 ? p.tiles : n_sm / 2;
    ffn_kernel<MODE, E><<<2 * pairs, kFfnThreads, ffn_smem(MODE), stream>>>(p);
    return cudaGetLastError();
}
template <int MODE> cudaError_t ffn_launch(const FfnParams &p, int dtype, int n_sm, cudaStream_t stream) {
    return dtype == 1 ? ffn_launch_typed<MODE, __half>(p, n_sm, stream)
                      : ffn_launch_typed<MODE, __nv_bfloat16>(p, n_sm, stream);
}

int ceil_div(long long a, int b) { return static_cast<int>((a + b - 1) / b); }

bool set_tiles(FfnParams &p, int tm, int tn) {
    if ((long long)tm * tn > (1 << 30)) return false;
    p.tm = make_fastdiv(tm);
    p.tiles = tm * tn;
    return true;
}

// Columns of the kDx and kDw tiles: 128 wastes fewer columns behind D, 256 reads each A block half as often.
int tile_columns(int D) { return D % 256 == 0 || D > 1024 ? 256 : 128; }

}  // namespace

bool ffn_supported(const FfnProblem &q) { return (q.dtype == 1 || q.dtype == 2) && tensor_map_encoder() != nullptr; }

cudaError_t launch_ffn(const FfnProblem &q, void *out, cudaStream_t stream) {
    int n_sm = 0;
    cudaError_t e = sm_count(&n_sm);
    if (e != cudaSuccess) return e;
    FfnParams p;
    std::memset(&p, 0, sizeof(p));
    if (!ffn_map(&p.a[0], q.x, q.dtype, q.M, q.D, q.x_stride, 128) ||
        !ffn_map(&p.b[0], q.w_gate, q.dtype, q.F, q.D, q.D, 128) ||
        !ffn_map(&p.b[1], q.w_value, q.dtype, q.F, q.D, q.D, 128) || !ffn_map(&p.o[0], out, q.dtype, q.M, q.F, q.F, 32) ||
        !set_tiles(p, ceil_div(q.M, kTileM), ceil_div(q.F, 128)))
        return cudaErrorInvalidValue;
    p.nk = ceil_div(q.D, kBlockK);
    p.rows = static_cast<int>(q.M);
    p.cols = q.F;
    p.bn = 256;
    p.idesc = instr_desc(q.dtype == 1 ? kFmtF16 : kFmtBF16, kTileM, 256, 0, 0);
    return ffn_launch<kFwd>(p, q.dtype, n_sm, stream);
}

size_t ffn_bwd_workspace(long long M, int F) { return ((size_t)M * F * 2 + 255) / 256 * 256 * 2; }

cudaError_t launch_ffn_bwd(const FfnProblem &q, const void *dout, long long dout_stride, void *dx, void *dw_gate,
                           void *dw_value, void *workspace, cudaStream_t stream) {
    int n_sm = 0;
    cudaError_t e = sm_count(&n_sm);
    if (e != cudaSuccess) return e;
    char *dg = static_cast<char *>(workspace), *dv = dg + ffn_bwd_workspace(q.M, q.F) / 2;
    const uint32_t fmt = q.dtype == 1 ? kFmtF16 : kFmtBF16;
    FfnParams p;
    std::memset(&p, 0, sizeof(p));
    if (!ffn_map(&p.a[0], q.x, q.dtype, q.M, q.D, q.x_stride, 128) ||
        !ffn_map(&p.b[0], q.w_gate, q.dtype, q.F, q.D, q.D, 128) ||
        !ffn_map(&p.b[1], q.w_value, q.dtype, q.F, q.D, q.D, 128) || !ffn_map(&p.o[0], dg, q.dtype, q.M, q.F, q.F, 32) ||
        !ffn_map(&p.o[1], dv, q.dtype, q.M, q.F, q.F, 32) || !ffn_map(&p.dh, dout, q.dtype, q.M, q.F, dout_stride, 32) ||
        !set_tiles(p, ceil_div(q.M, kTileM), ceil_div(q.F, 128)))
        return cudaErrorInvalidValue;
    p.nk = ceil_div(q.D, kBlockK);
    p.rows = static_cast<int>(q.M);
    p.cols = q.F;
    p.bn = 256;
    p.idesc = instr_desc(fmt, kTileM, 256, 0, 0);
    if ((e = ffn_launch<kAct>(p, q.dtype, n_sm, stream)) != cudaSuccess) return e;

    const int bn = tile_columns(q.D);
    std::memset(&p, 0, sizeof(p));
    if (!ffn_map(&p.a[0], dg, q.dtype, q.M, q.F, q.F, 128) || !ffn_map(&p.a[1], dv, q.dtype, q.M, q.F, q.F, 128) ||
        !ffn_map(&p.b[0], q.w_gate, q.dtype, q.F, q.D, q.D, 64) || !ffn_map(&p.b[1], q.w_value, q.dtype, q.F, q.D, q.D, 64) ||
        !ffn_map(&p.o[0], dx, q.dtype, q.M, q.D, q.D, 32) || !set_tiles(p, ceil_div(q.M, kTileM), ceil_div(q.D, bn)))
        return cudaErrorInvalidValue;
    p.nk_half = ceil_div(q.F, kBlockK);
    p.nk = 2 * p.nk_half;
    p.rows = static_cast<int>(q.M);
    p.cols = q.D;
    p.bn = bn;
    p.idesc = instr_desc(fmt, kTileM, bn, 0, 1);
    if ((e = ffn_launch<kDx>(p, q.dtype, n_sm, stream)) != cudaSuccess) return e;

    std::memset(&p, 0, sizeof(p));
    if (!ffn_map(&p.a[0], dg, q.dtype, q.M, q.F, q.F, 64) || !ffn_map(&p.a[1], dv, q.dtype, q.M, q.F, q.F, 64) ||
        !ffn_map(&p.b[0], q.x, q.dtype, q.M, q.D, q.x_stride, 64) || !ffn_map(&p.o[0], dw_gate, q.dtype, q.F, q.D, q.D, 32) ||
        !ffn_map(&p.o[1], dw_value, q.dtype, q.F, q.D, q.D, 32) || !set_tiles(p, 2 * ceil_div(q.F, kTileM), ceil_div(q.D, bn)))
        return cudaErrorInvalidValue;
    p.nk = ceil_div(q.M, kBlockK);
    p.rows = q.F;
    p.cols = q.D;
    p.bn = bn;
    p.idesc = instr_desc(fmt, kTileM, bn, 1, 1);
    return ffn_launch<kDw>(p, q.dtype, n_sm, stream);
}

cudaError_t read_and_clear_ffn_status(unsigned int *status) {
    cudaError_t e = cudaMemcpyFromSymbol(status, g_ffn_status, sizeof(unsigned int));
    if (e != cudaSuccess) return e;
    const unsigned int zero = 0;
    return cudaMemcpyToSymbol(g_ffn_status, &zero, sizeof(unsigned int));
}

}  // namespace gtr
