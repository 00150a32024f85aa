// Product of 8-bit matrices whose values share a scale per 128 columns: y = x w^T + b, x [rows][width] with a scale for each row and
// block of columns, w [outs][width] with one for each 128 x 128 block.
//
// The tensor cores add up e4m3 products exactly as they are; a scale can only be applied to the sum of one block of 128 columns.  So
// the accumulator in tensor memory holds one such block (four K = 32 instructions) and is read back, multiplied by its scales and
// added to fp32 sums in registers while the next block is computed into a second accumulator.
#include "../../include/lstm_b200.h"
#include "operators.cuh"

#include <cuda.h>

namespace lstm {
namespace {

constexpr int kBlockK = 128;          // columns of a block: 128 bytes, one row of a swizzled tile
constexpr int kTileOuts = 128;        // rows of w in a tile: those of one block of scales

struct ProductArgs {
    int rows, outs, blocks;           // blocks of 128 columns
    int csize;                        // CTAs that share a tile, each with its own blocks of columns
    int stages;
    const float *sx, *sw, *bias;
    void *y;
    long long y_ld;
};

__device__ __forceinline__ void umma_e4m3(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// instruction descriptor: fp32 sums, e4m3 x e4m3, both K-major, M x N
__device__ constexpr uint32_t idesc_e4m3(int m, int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }

__device__ __forceinline__ uint32_t rank_in_cluster()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t at_rank(uint32_t smem_addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---------------------------------------------------------------------------------------------------
// Few rows of x: bound by the bytes of w.  128 rows of w are the M operand, R rows of x the N operand, and the blocks of columns
// are split over a cluster of up to eight CTAs so that all SMs read; their sums meet in distributed shared memory, in one order.
// Warps 0-3 read the accumulators back (quadrant = warp), warp 4 fetches, warp 5 multiplies.
// ---------------------------------------------------------------------------------------------------
constexpr int kFewThreads = 192;
constexpr int kMaxStages = 12;

template <typename T, int R>
__global__ void __launch_bounds__(kFewThreads)
fp8_few_rows_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ ProductArgs p)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long full_bar[kMaxStages], empty_bar[kMaxStages], sums_full[2], sums_empty[2];
    __shared__ __align__(16) float scale[2][R];
    __shared__ uint32_t tmem_base_s;
    __shared__ int abort_s;
    constexpr uint32_t kWBytes = kTileOuts * kBlockK, kStage = kWBytes + R * kBlockK;
    constexpr uint32_t kCols = 2 * R < 32 ? 32 : 2 * R;

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int rank = p.csize > 1 ? (int)rank_in_cluster() : 0;
    const int n_tile = blockIdx.x / p.csize, m0 = blockIdx.y * R;
    const int j0 = (int)((long long)rank * p.blocks / p.csize), nj = (int)((long long)(rank + 1) * p.blocks / p.csize) - j0;
    const uint32_t tiles = (smem_u32(smem_raw) + 1023u) & ~1023u;

    if (tid == 0) {
        abort_s = 0;
        for (int s = 0; s < p.stages; ++s) { mbar_init(smem_u32(&full_bar[s]), 1); mbar_init(smem_u32(&empty_bar[s]), 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(smem_u32(&sums_full[s]), 1); mbar_init(smem_u32(&sums_empty[s]), 4); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "r"(kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = tmem_base_s;
    volatile int *abort_flag = &abort_s;

    float sum[R];
    if (warp == 4) {
        if (lane == 0) {
            int s = 0;
            uint32_t ph = 0;
            for (int i = 0; i < nj; ++i) {
                if (!mbar_wait(smem_u32(&empty_bar[s]), ph ^ 1u, abort_flag)) break;
                const uint32_t fb = smem_u32(&full_bar[s]), at = tiles + (uint32_t)s * kStage;
                mbar_expect_tx(fb, kStage);
                tma_load_2d(at, &map_w, fb, (j0 + i) * kBlockK, n_tile * kTileOuts);
                tma_load_2d(at + kWBytes, &map_x, fb, (j0 + i) * kBlockK, m0);
                if (++s == p.stages) { s = 0; ph ^= 1u; }
            }
        }
    } else if (warp == 5) {
        int s = 0;
        uint32_t ph = 0;
        for (int i = 0; i < nj; ++i) {
            const int buf = i & 1;
            bool ok = mbar_wait(smem_u32(&sums_empty[buf]), ((i >> 1) & 1) ^ 1u, abort_flag);
            ok = ok && mbar_wait(smem_u32(&full_bar[s]), ph, abort_flag);
            if (!__all_sync(0xffffffffu, ok)) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t at = tiles + (uint32_t)s * kStage;
            const uint64_t wdesc = umma_desc_sw128(at), xdesc = umma_desc_sw128(at + kWBytes);
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < kBlockK / 32; ++k)
                    umma_e4m3(tmem_base + buf * R, wdesc + 2 * k, xdesc + 2 * k, idesc_e4m3(kTileOuts, R), k > 0);
                umma_commit(smem_u32(&empty_bar[s]));
                umma_commit(smem_u32(&sums_full[buf]));
            }
            __syncwarp();
            if (++s == p.stages) { s = 0; ph ^= 1u; }
        }
    } else {
        // thread = one row of w; the scales of the R rows of x, times the block's scale of w, lie in shared memory
#pragma unroll
        for (int r = 0; r < R; ++r) sum[r] = 0.0f;
        const bool mine = tid < R && m0 + tid < p.rows;
        const float *sx = p.sx + (long long)(m0 + tid) * p.blocks + j0, *sw = p.sw + (long long)n_tile * p.blocks + j0;
        float next = mine && nj > 0 ? sx[0] * sw[0] : 0.0f;
        bool ok = true;
        for (int i = 0; i < nj; ++i) {
            const int buf = i & 1;
            if (tid < R) scale[buf][tid] = next;
            bar_sync(1, 128);                            // the other buffer is written next when all have left it
            if (mine && i + 1 < nj) next = sx[i + 1] * sw[i + 1];
            ok = mbar_wait(smem_u32(&sums_full[buf]), (i >> 1) & 1, abort_flag) && ok;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            __syncwarp();
#pragma unroll
            for (int c = 0; c < R; c += 16) {
                uint32_t v[16];
                tmem_ld16(tmem_base + ((uint32_t)(warp * 32) << 16) + (uint32_t)(buf * R + c), v);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                for (int k = 0; k < 16; ++k) sum[c + k] = fmaf(__uint_as_float(v[k]), scale[buf][c + k], sum[c + k]);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sums_empty[buf]));
        }
        if (!ok) {
#pragma unroll
            for (int r = 0; r < R; ++r) sum[r] = __uint_as_float(0x7fffffffu);
        }
    }

    const int n = n_tile * kTileOuts + tid;
    T *y = (T *)p.y;
    if (p.csize > 1) {
        // all blocks have been multiplied: the stages' memory takes this CTA's sums
        float *part = reinterpret_cast<float *>(smem_raw + (tiles - smem_u32(smem_raw)));
        if (warp < 4) {
#pragma unroll
            for (int r = 0; r < R; ++r) part[r * kTileOuts + tid] = sum[r];
        }
        cluster_sync();
        if (warp < 4 && n < p.outs) {
            const float b = p.bias ? p.bias[n] : 0.0f;
            const uint32_t here = tiles + (uint32_t)tid * 4;
            for (int r = rank; r < R && m0 + r < p.rows; r += p.csize) {
                float v = 0.0f;
                for (int c = 0; c < p.csize; ++c) {
                    float u;
                    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(u) : "r"(at_rank(here + r * kTileOuts * 4, c)) : "memory");
                    v += u;
                }
                y[(long long)(m0 + r) * p.y_ld + n] = T(v + b);
            }
        }
        cluster_sync();                                  // nobody's memory goes while another reads it
    } else if (warp < 4 && n < p.outs) {
        const float b = p.bias ? p.bias[n] : 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (m0 + r < p.rows) y[(long long)(m0 + r) * p.y_ld + n] = T(sum[r] + b);
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 5) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kCols) : "memory");
    }
}

template <typename T, int R>
cudaError_t launch_few(ProductArgs &p, const CUtensorMap &mw, const CUtensorMap &mx, int sms, cudaStream_t st)
{
    const void *fn = (const void *)fp8_few_rows_kernel<T, R>;
    const int n_tiles = (p.outs + kTileOuts - 1) / kTileOuts, m_tiles = (p.rows + R - 1) / R;
    const long long tiles = (long long)n_tiles * m_tiles;
    p.csize = (int)(sms / tiles < 1 ? 1 : sms / tiles > 8 ? 8 : sms / tiles);
    if (p.csize > p.blocks) p.csize = p.blocks;
    constexpr int kStage = kTileOuts * kBlockK + R * kBlockK;
    // two CTAs of an SM share its memory; the sums of a split tile need the first R / 32 stages' worth
    int stages = 108 * 1024 / kStage;
    if (stages > kMaxStages) stages = kMaxStages;
    const int most = (p.blocks + p.csize - 1) / p.csize, least = (R * kTileOuts * 4 + kStage - 1) / kStage;
    if (stages > most) stages = most;
    if (stages < least) stages = least;
    p.stages = stages;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(n_tiles * p.csize), (unsigned)m_tiles);
    cfg.blockDim = dim3(kFewThreads);
    cfg.dynamicSmemBytes = (size_t)stages * kStage + 1024;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = p.csize;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = p.csize > 1 ? 1 : 0;
    cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cfg.dynamicSmemBytes);
    if (e != cudaSuccess) return e;
    void *args[] = {(void *)&mw, (void *)&mx, &p};
    return cudaLaunchKernelExC(&cfg, fn, args);
}

template <typename T>
cudaError_t launch(ProductArgs &p, const void *qx, long long qx_ld, const void *qw, long long qw_ld, int width, int sms, cudaStream_t st, bool &mapped)
{
    const int R = p.rows <= 16 ? 16 : p.rows <= 32 ? 32 : p.rows <= 64 ? 64 : 128;
    CUtensorMap mw, mx;
    mapped = encode_tmap_2d(&mw, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, qw, p.outs, width, qw_ld, kTileOuts) &&
             encode_tmap_2d(&mx, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, qx, p.rows, width, qx_ld, R);
    if (!mapped) return cudaErrorInvalidValue;
    if (R == 16) return launch_few<T, 16>(p, mw, mx, sms, st);
    if (R == 32) return launch_few<T, 32>(p, mw, mx, sms, st);
    if (R == 64) return launch_few<T, 64>(p, mw, mx, sms, st);
    return launch_few<T, 128>(p, mw, mx, sms, st);
}

}  // namespace
}  // namespace lstm

using namespace lstm;

extern "C" int lstm_fp8_product(const void *qx, long long qx_ld, const float *sx, const void *qw, long long qw_ld, const float *sw, const float *bias,
                                int rows, int outs, int width, int dtype, void *y, long long y_ld, void *cuda_stream, char *err, int errlen)
{
    const Failure fail{err, errlen};
    if (rows < 0 || outs < 0 || width < 1) return fail(LSTM_ERR_INVALID, "bad argument: rows and outs must be 0 or more, width 1 or more");
    if (!known_type(dtype)) return fail(LSTM_ERR_INVALID, "bad argument: dtype must be LSTM_F32 or LSTM_BF16");
    if (rows == 0 || outs == 0) return LSTM_OK;
    if (!qx || !sx || !qw || !sw || !y) return fail(LSTM_ERR_INVALID, "bad argument: qx, sx, qw, sw and y must be given");
    if (!aligned_to(sx, 4) || !aligned_to(sw, 4) || !aligned_to(bias, 4) || !aligned_to(y, bytes_of(dtype)))
        return fail(LSTM_ERR_INVALID, "bad argument: a pointer is not aligned to its elements");
    if (!aligned_to(qx, 16) || !aligned_to(qw, 16) || qx_ld % 16 || qw_ld % 16 || qx_ld < width || qw_ld < width)
        return fail(LSTM_ERR_INVALID, "bad argument: 8-bit rows must start on 16 bytes and not overlap");
    if (rows > 65535 * 128) return fail(LSTM_ERR_UNSUPPORTED, "more than 65535 tiles of rows");
    int sms = 0;
    if (const int rc = device_sms(sms, fail)) return rc;
    ProductArgs p = {};
    p.rows = rows; p.outs = outs; p.blocks = (width + kBlockK - 1) / kBlockK;
    p.sx = sx; p.sw = sw; p.bias = bias;
    p.y = y; p.y_ld = y_ld;
    bool mapped = true;
    const cudaError_t e = dtype == LSTM_BF16 ? launch<__nv_bfloat16>(p, qx, qx_ld, qw, qw_ld, width, sms, (cudaStream_t)cuda_stream, mapped)
                                             : launch<float>(p, qx, qx_ld, qw, qw_ld, width, sms, (cudaStream_t)cuda_stream, mapped);
    if (!mapped) return fail(LSTM_ERR_CUDA, "the tensor maps of the operands could not be made");
    return e == cudaSuccess ? LSTM_OK : fail.cuda(e);
}
