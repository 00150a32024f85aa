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
    int stored;                       // y is written by tensor copies (its rows start and end on 16 bytes)
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

// mbar_wait by warps that have nothing else to do: each try may sleep for some microseconds, so that they leave the scheduler to others
__device__ __forceinline__ bool wait_long(uint32_t bar, uint32_t parity, volatile int *abort_flag)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity), "r"(10000u) : "memory");
    return ok ? true : mbar_wait(bar, parity, abort_flag);
}
// the values of a read-back are there behind this
__device__ __forceinline__ void tmem_arrived(uint32_t (&v)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]),
                   "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])::"memory");
}

// A fetching thread that gives up lets its copies in flight land (microseconds; this is milliseconds) before the CTA's memory goes.
__device__ __forceinline__ void let_copies_land()
{
    for (int i = 0; i < 4; ++i) __nanosleep(1000000);
}

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
// One row x 6000 x 1500 takes 5.3 us, 16 rows 6.0, one row x 8192 x 8192 (10.3 us of bytes) 15.5: a launch and its fill (tensor memory, maps,
// first bytes) are 3 to 4 us of each.
// ---------------------------------------------------------------------------------------------------
constexpr int kFewThreads = 192;
constexpr int kFewSmem = 108 * 1024;
constexpr int kMaxStages = 12;
constexpr int kMaxSplit = 8;          // CTAs that share a tile

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
                if (!mbar_wait(smem_u32(&empty_bar[s]), ph ^ 1u, abort_flag)) { let_copies_land(); break; }
                const uint32_t fb = smem_u32(&full_bar[s]), at = tiles + (uint32_t)s * kStage;
                mbar_expect_tx(fb, kStage);
                tma_load_2d(at, &map_w, fb, (j0 + i) * kBlockK, n_tile * kTileOuts);
                tma_load_2d(at + kWBytes, &map_x, fb, (j0 + i) * kBlockK, m0);
                if (++s == p.stages) { s = 0; ph ^= 1u; }
            }
        }
        __syncwarp();
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
        float next_x = mine && nj > 0 ? sx[0] : 0.0f, next_w = nj > 0 ? sw[0] : 0.0f;
        bool ok = true;
        for (int i = 0; i < nj; ++i) {
            const int buf = i & 1;
            if (tid < R) scale[buf][tid] = next_x * next_w;
            bar_sync(1, 128);                            // the other buffer is written next when all have left it
            if (mine && i + 1 < nj) { next_x = sx[i + 1]; next_w = sw[i + 1]; }
            ok = mbar_wait(smem_u32(&sums_full[buf]), (i >> 1) & 1, abort_flag) && ok;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            __syncwarp();
#pragma unroll
            for (int c = 0; c < R; c += 16) {
                uint32_t v[16];
                tmem_ld16(tmem_base + ((uint32_t)(warp * 32) << 16) + (uint32_t)(buf * R + c), v);
                tmem_arrived(v);
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
        // all blocks have been multiplied: the stages' memory takes this CTA's sums, four rows of x side by side for each row of w
        float4 *part = reinterpret_cast<float4 *>(smem_raw + (tiles - smem_u32(smem_raw)));
        if (warp < 4) {
#pragma unroll
            for (int r = 0; r < R; r += 4) part[r / 4 * kTileOuts + tid] = make_float4(sum[r], sum[r + 1], sum[r + 2], sum[r + 3]);
        }
        cluster_sync();
        if (warp < 4 && n < p.outs) {
            const float b = p.bias ? p.bias[n] : 0.0f;
            const uint32_t here = tiles + (uint32_t)tid * 16;
            for (int q = rank; q < R / 4 && m0 + 4 * q < p.rows; q += p.csize) {
                float4 u[kMaxSplit];                     // all on their way before the first is added
#pragma unroll
                for (int c = 0; c < kMaxSplit; ++c)
                    if (c < p.csize)
                        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                                     : "=f"(u[c].x), "=f"(u[c].y), "=f"(u[c].z), "=f"(u[c].w) : "r"(at_rank(here + q * kTileOuts * 16, c)) : "memory");
                float v[4] = {u[0].x, u[0].y, u[0].z, u[0].w};
#pragma unroll
                for (int c = 1; c < kMaxSplit; ++c)
                    if (c < p.csize) { v[0] += u[c].x; v[1] += u[c].y; v[2] += u[c].z; v[3] += u[c].w; }
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (m0 + 4 * q + k < p.rows) y[(long long)(m0 + 4 * q + k) * p.y_ld + n] = T(v[k] + b);
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
    // CTAs for one and a half of the SMs: with fewer some SMs read nothing, with more the joining costs more than their reading saves
    // (64 x 6000 x 1500: 3 CTAs a tile 13.4 us, 4 10.6, 6 20.2)
    const long long share = 3ll * sms / (2 * tiles);
    p.csize = (int)(share < 1 ? 1 : share > kMaxSplit ? kMaxSplit : share);
    if (p.csize > p.blocks) p.csize = p.blocks;
    constexpr int kStage = kTileOuts * kBlockK + R * kBlockK;
    // two CTAs of an SM share its memory; the sums of a split tile need the first R / 32 stages' worth
    int stages = kFewSmem / kStage;
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
    static std::atomic<unsigned long long> prepared;
    const cudaError_t e = prepare_kernel(fn, prepared, kFewSmem + 1024, false);
    if (e != cudaSuccess) return e;
    void *args[] = {(void *)&mw, (void *)&mx, &p};
    return cudaLaunchKernelExC(&cfg, fn, args);
}

// ---------------------------------------------------------------------------------------------------
// Many rows of x: bound by the tensor cores, and by what brings operands to them.  A pair of CTAs (two SMs) multiplies 256 rows of x
// by 256 rows of w at a time: each holds 128 rows of x and half of the rows of w, which the pair's instruction reads from both, so
// that a block costs 32 KB from L2 for each 128 x 256 sums.  Rows of x are the lanes of the accumulator: a thread's sums share
// one scale of x and one of w, one multiply-add an element.  The pairs stay and walk over the tiles.  A block is multiplied in two
// halves of its columns with barriers of their own, so that four accumulators are on their way between the tensor cores and
// the warps that read them.
// Warps 0-15 read the accumulators back (quadrant = warp % 4, 64 columns each), warp 16 fetches, warp 17 of the first
// CTA multiplies for both, warps 18 and 19 bring the scales of the rows of x, which lie a row's length apart, 16 blocks at a time into
// shared memory (each reading warp on its own would touch 32 lines a block).
// 25600 x 6400 x 1600 in 278 to 284 us: 1850 TFLOP/s, the tensor pipe 49 % active (in a burst; for seconds under the power cap 323, a bf16 product of
// that size 357 and 412).  Of those 206 are operands and products (without reading
// back), 50 the reading back, the rest the tiles' ends.  Steps: eight reading warps with 128 sums each 704 us, 16 with 64 410, scales staged and
// results turned in shared memory 306, tensor copies of the results 284.
// ---------------------------------------------------------------------------------------------------
constexpr int kPairRows = 256, kPairOuts = 256;
constexpr int kPairThreads = 640;
constexpr int kPairCols = 64;                                       // columns of a warp
constexpr int kPairStages = 4;
constexpr uint32_t kHalfTile = 128 * kBlockK;                       // 128 rows of either operand
constexpr int kTurnPitch = 34, kTurn = 32 * kTurnPitch;             // words in which a warp turns 32 rows of 32 words (64 bf16 or 32 fp32)
constexpr int kScaleBlocks = 16, kScalePitch = 130;                 // scales staged at once, [block][row]: eight rows x four words without conflicts
constexpr int kScales = kScaleBlocks * kScalePitch + kPairOuts;     // and the tile's biases
constexpr int kPairSmem = kPairStages * 2 * kHalfTile + (16 * kTurn + 2 * kScales) * 4;

__device__ __forceinline__ void umma_e4m3_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// arrives on the barrier at this place in both CTAs once the instructions issued so far have run
__device__ __forceinline__ void umma_commit_pair(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// a tile into this CTA's memory, counted by a barrier that may be the other CTA's
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// sum += v * scale, two to an instruction
__device__ __forceinline__ void add_scaled(float &s0, float &s1, uint32_t v0, uint32_t v1, float scale)
{
    asm("{\n\t.reg .b64 s, v, k;\n\tmov.b64 s, {%0, %1};\n\tmov.b64 v, {%2, %3};\n\tmov.b64 k, {%4, %4};\n\t"
        "fma.rn.f32x2 s, v, k, s;\n\tmov.b64 {%0, %1}, s;\n\t}"
        : "+f"(s0), "+f"(s1) : "r"(v0), "r"(v1), "f"(scale));
}

template <typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
fp8_many_rows_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_y,
                     const __grid_constant__ ProductArgs p)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long full_bar[kPairStages], empty_bar[kPairStages], sums_full[4], sums_empty[4], scales_full[2], scales_empty[2];
    __shared__ uint32_t tmem_base_s;
    __shared__ int abort_s;

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int rank = (int)rank_in_cluster();
    const uint32_t tiles = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int n_tiles = (p.outs + kPairOuts - 1) / kPairOuts;
    const long long all = (long long)n_tiles * ((p.rows + kPairRows - 1) / kPairRows);
    const int pairs = gridDim.x / 2, pair = blockIdx.x / 2;

    if (tid == 0) {
        abort_s = 0;
        for (int s = 0; s < kPairStages; ++s) { mbar_init(smem_u32(&full_bar[s]), 1); mbar_init(smem_u32(&empty_bar[s]), 1); }
        for (int s = 0; s < 4; ++s) { mbar_init(smem_u32(&sums_full[s]), 1); mbar_init(smem_u32(&sums_empty[s]), 16); }
        for (int s = 0; s < 2; ++s) { mbar_init(smem_u32(&scales_full[s]), 64); mbar_init(smem_u32(&scales_empty[s]), 16); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 17) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();                                      // both CTAs' barriers and tensor memory are there
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = tmem_base_s;
    volatile int *abort_flag = &abort_s;
    unsigned char *behind = smem_raw + (tiles - smem_u32(smem_raw)) + kPairStages * 2 * kHalfTile;       // a multiple of 1024 bytes
    float *staged = reinterpret_cast<float *>(behind + 16 * kTurn * 4);

    if (warp >= 18) {
        // rows 64 (warp - 18) and on: lane = row of eight, word of four
        int c = 0;
        bool ok = true;
        for (long long tile = pair; tile < all && ok; tile += pairs) {
            const int m0 = (int)(tile / n_tiles) * kPairRows + rank * 128, r0 = (warp - 18) * 64 + (lane >> 2);
            for (int j0 = 0; j0 < p.blocks; j0 += kScaleBlocks, ++c) {
                if (!(ok = mbar_wait(smem_u32(&scales_empty[c & 1]), (uint32_t)((c >> 1) & 1) ^ 1u, abort_flag))) break;
                float *to = staged + (c & 1) * kScales;
#pragma unroll 2
                for (int r = r0; r < r0 + 64; r += 8) {
                    const float *from = p.sx + (long long)(m0 + r) * p.blocks;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int j = 4 * (lane & 3) + k;
                        to[j * kScalePitch + r] = m0 + r < p.rows && j0 + j < p.blocks ? from[j0 + j] : 0.0f;
                    }
                }
                if (warp == 18 && j0 == 0) {             // the biases come with a tile's first scales
                    const int n0 = (int)(tile % n_tiles) * kPairOuts;
#pragma unroll
                    for (int n = lane; n < kPairOuts; n += 32)
                        to[kScaleBlocks * kScalePitch + n] = p.bias && n0 + n < p.outs ? p.bias[n0 + n] : 0.0f;
                }
                mbar_arrive(smem_u32(&scales_full[c & 1]));
            }
        }
        __syncwarp();
    } else if (warp == 16) {
        if (lane == 0) {
            int s = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (long long tile = pair; tile < all && ok; tile += pairs) {
                const int m0 = (int)(tile / n_tiles) * kPairRows + rank * 128, n0 = (int)(tile % n_tiles) * kPairOuts + rank * 128;
                for (int j = 0; j < p.blocks; ++j) {
                    if (!(ok = mbar_wait(smem_u32(&empty_bar[s]), ph ^ 1u, abort_flag))) { let_copies_land(); break; }
                    const uint32_t at = tiles + (uint32_t)s * 2 * kHalfTile, fb = at_rank(smem_u32(&full_bar[s]), 0);
                    if (rank == 0) mbar_expect_tx(smem_u32(&full_bar[s]), 4 * kHalfTile);      // both CTAs' tiles
                    tma_load_2d_pair(at, &map_x, fb, j * kBlockK, m0);
                    tma_load_2d_pair(at + kHalfTile, &map_w, fb, j * kBlockK, n0);
                    if (++s == kPairStages) { s = 0; ph ^= 1u; }
                }
            }
        }
        __syncwarp();
    } else if (warp == 17) {
        if (rank == 0) {
            int s = 0;
            uint32_t ph = 0;
            long long i = 0;
            bool ok = true;
            for (long long tile = pair; tile < all && ok; tile += pairs) {
                for (int j = 0; j < p.blocks; ++j, ++i) {
                    const int buf = (int)(i & 1);
                    if (!(ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&full_bar[s]), ph, abort_flag)))) break;
                    const uint32_t at = tiles + (uint32_t)s * 2 * kHalfTile;
                    const uint64_t xdesc = umma_desc_sw128(at), wdesc = umma_desc_sw128(at + kHalfTile);
#pragma unroll
                    for (int half = 0; half < 2 && ok; ++half) {
                        const int set = 2 * buf + half;
                        if (!(ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sums_empty[set]), (uint32_t)((i >> 1) & 1) ^ 1u, abort_flag)))) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < kBlockK / 32; ++k)
                                umma_e4m3_pair(tmem_base + set * (kPairOuts / 2), xdesc + 2 * k, wdesc + half * (kHalfTile / 2 / 16) + 2 * k,
                                               idesc_e4m3(kPairRows, kPairOuts / 2), k > 0);
                            if (half == 1) umma_commit_pair(smem_u32(&empty_bar[s]));
                            umma_commit_pair(smem_u32(&sums_full[set]));
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    __syncwarp();
                    if (++s == kPairStages) { s = 0; ph ^= 1u; }
                }
            }
        }
    } else {
        // a half's 128 columns of tensor memory are 64 rows of w from each CTA
        const int quad = warp & 3, part = warp >> 2, col0 = (part & 1) * 128 + (part >> 1) * 64;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        uint32_t *turn = reinterpret_cast<uint32_t *>(behind) + warp * (p.stored ? 32 * 32 : kTurn);
        T *y = (T *)p.y;
        constexpr int kWord = 4 / sizeof(T);                        // columns of a word
        // words that may be stored at once: two, one, or (rows of bf16 that start anywhere) half of one
        const unsigned long long off = (unsigned long long)y | (unsigned long long)p.y_ld * sizeof(T);
        const int wide = off % 8 == 0 ? 2 : off % 4 == 0 ? 1 : 0;
        // this half's barriers: of the accumulators of even blocks, those of odd ones 16 bytes on
        const uint32_t full_at = smem_u32(&sums_full[part >> 1]), empty_at = at_rank(smem_u32(&sums_empty[part >> 1]), 0);
        // columns of tensor memory: buffer, half, the warp's 64
        const uint32_t from0 = tmem_base + lanes + (uint32_t)(part * kPairCols);
        int chunk = 0;
        uint32_t i = 0;
        bool ok = true;
        for (long long tile = pair; tile < all; tile += pairs) {
            const int m0 = (int)(tile / n_tiles) * kPairRows + rank * 128 + quad * 32, n0 = (int)(tile % n_tiles) * kPairOuts + col0;
            const float *sw = p.sw + (long long)(n0 < p.outs ? n0 / kTileOuts : 0) * p.blocks;
            float sum[kPairCols], next_w = sw[0];
            for (int j0 = 0; j0 < p.blocks; j0 += kScaleBlocks, ++chunk) {
                ok = wait_long(smem_u32(&scales_full[chunk & 1]), (uint32_t)((chunk >> 1) & 1), abort_flag) && ok;
                const float *sx = staged + (chunk & 1) * kScales + quad * 32 + lane;
                if (j0 == 0) {
                    const float *bias = staged + (chunk & 1) * kScales + kScaleBlocks * kScalePitch + col0;
#pragma unroll
                    for (int c = 0; c < kPairCols; c += 4) {
                        const float4 b = *reinterpret_cast<const float4 *>(bias + c);
                        sum[c] = b.x; sum[c + 1] = b.y; sum[c + 2] = b.z; sum[c + 3] = b.w;
                    }
                }
                const int j1 = min(j0 + kScaleBlocks, p.blocks);
                for (int j = j0; j < j1; ++j, ++i, sx += kScalePitch) {
                    const float scale = *sx * next_w;
                    if (j + 1 < p.blocks) next_w = sw[j + 1];
                    const uint32_t set = 2 * (i & 1);
                    ok = wait_long(full_at + 8 * set, (i >> 1) & 1, abort_flag) && ok;
                    __syncwarp();
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t from = from0 + set * (kPairOuts / 2);
                    uint32_t v[2][16];
                    tmem_ld16(from, v[0]);
#pragma unroll
                    for (int c = 0; c < kPairCols; c += 16) {
                        const int now = c / 16 & 1;
                        tmem_arrived(v[now]);
                        if (c + 16 < kPairCols) tmem_ld16(from + c + 16, v[now ^ 1]);
                        else {
                            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                            __syncwarp();
                            if (lane == 0) mbar_arrive_cluster(empty_at + 8 * set);
                        }
#pragma unroll
                        for (int k = 0; k < 16; k += 2) add_scaled(sum[c + k], sum[c + k + 1], v[now][k], v[now][k + 1], scale);
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&scales_empty[chunk & 1]));
            }
            if (!ok) {
#pragma unroll
                for (int c = 0; c < kPairCols; ++c) sum[c] = __uint_as_float(0x7fffffffu);
            }
            // A thread has a row, memory wants columns side by side: 32 rows of 128 bytes go through shared memory, from where a tensor
            // copy takes them (and leaves out what lies outside of y) while the warp goes on ...
            if (p.stored) {
#pragma unroll
                for (int c0 = 0; c0 < kPairCols; c0 += 32 * kWord) {
                    if (n0 + c0 >= p.outs || m0 >= p.rows) break;
                    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 8; ++j)          // 16 bytes, in the swizzle's place
                        *reinterpret_cast<Vec<T, 4 * kWord> *>(turn + lane * 32 + (j ^ (lane & 7)) * 4) = to_vec<T, 4 * kWord>(&sum[c0 + j * 4 * kWord]);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];"
                                     ::"l"(&map_y), "r"(n0 + c0), "r"(m0), "r"(smem_u32(turn)) : "memory");
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                }
                continue;
            }
            // ... or, where rows start anywhere, 32 x 32 words at a time change places within the warp
            const int rows = min(32, p.rows - m0);
#pragma unroll
            for (int c0 = 0; c0 < kPairCols; c0 += 32 * kWord) {
                const int left = p.outs - n0 - c0;
                if (left <= 0 || rows <= 0) break;
                __syncwarp();
#pragma unroll
                for (int w = 0; w < 32; w += 2) {
                    *reinterpret_cast<Vec<T, 2 * kWord> *>(turn + lane * kTurnPitch + w) = to_vec<T, 2 * kWord>(&sum[c0 + w * kWord]);
                }
                __syncwarp();
                T *out = y + (long long)m0 * p.y_ld + n0 + c0;
                if (wide == 2 && left >= 32 * kWord) {
                    const int w = 2 * (lane & 15), r0 = lane >> 4;
                    out += r0 * p.y_ld + w * kWord;
#pragma unroll
                    for (int r = 0; r < 32; r += 2, out += 2 * p.y_ld)
                        if (r + r0 < rows) *reinterpret_cast<uint2 *>(out) = *reinterpret_cast<const uint2 *>(turn + (r + r0) * kTurnPitch + w);
                } else if (wide && left >= 32 * kWord) {
                    out += lane * kWord;
#pragma unroll 8
                    for (int r = 0; r < rows; ++r, out += p.y_ld) *reinterpret_cast<uint32_t *>(out) = turn[r * kTurnPitch + lane];
                } else {
                    for (int c = lane; c < 32 * kWord && c < left; c += 32) {
                        T *o = out + c;
#pragma unroll 8
                        for (int r = 0; r < rows; ++r, o += p.y_ld) *o = reinterpret_cast<const T *>(turn + r * kTurnPitch)[c];
                    }
                }
            }
        }
        if (p.stored && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        __syncwarp();
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();                                      // no barrier and no operand goes while the other CTA needs it
    if (warp == 17) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    }
}

template <typename T>
cudaError_t launch_many(ProductArgs &p, const CUtensorMap &mw, const CUtensorMap &mx, int sms, cudaStream_t st)
{
    CUtensorMap my = mx;
    const int es = (int)sizeof(T);
    // (a row whose length is no multiple of 16 bytes would be written up to the next one)
    p.stored = aligned_to(p.y, 16) && p.y_ld * es % 16 == 0 && (long long)p.outs * es % 16 == 0 && p.y_ld >= p.outs &&
               encode_tmap_2d(&my, es == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, es, p.y, p.rows, p.outs, p.y_ld, 32);
    const void *fn = (const void *)fp8_many_rows_kernel<T>;
    static std::atomic<unsigned long long> prepared;
    const cudaError_t e = prepare_kernel(fn, prepared, kPairSmem + 1024, false);
    if (e != cudaSuccess) return e;
    const long long tiles = (long long)((p.outs + kPairOuts - 1) / kPairOuts) * ((p.rows + kPairRows - 1) / kPairRows);
    const int pairs = (int)(tiles < sms / 2 ? tiles : sms / 2);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * pairs));
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = kPairSmem + 1024;
    cfg.stream = st;
    void *args[] = {(void *)&mw, (void *)&mx, (void *)&my, &p};
    return cudaLaunchKernelExC(&cfg, fn, args);
}

template <typename T>
cudaError_t launch(ProductArgs &p, const void *qx, long long qx_ld, const void *qw, long long qw_ld, int width, int sms, cudaStream_t st, bool &mapped)
{
    const int R = p.rows <= 16 ? 16 : p.rows <= 32 ? 32 : p.rows <= 64 ? 64 : 128;
    // Pairs of CTAs from 64 tiles of 128 x 128 on.  us, few rows / pairs: 47 tiles (128 x 6000 x 1500) 11.1 / 11.9, 48 (700 x 1000 x 1500)
    // 11.2 / 12.5, 64 (1000 x 1000 x 1500) 13.0 / 12.6, 94 (160 x 6000 x 1500) 14.1 / 11.9, 96 (400 x 3000 x 6000) 28.5 / 28.2, 192 (1000 x 3000
    // x 6000) 49 / 30
    const bool many = p.rows > 128 && (p.rows + 127ll) / 128 * ((p.outs + 127ll) / 128) >= 64;
    CUtensorMap mw, mx;
    mapped = encode_tmap_2d(&mw, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, qw, p.outs, width, qw_ld, kTileOuts) &&
             encode_tmap_2d(&mx, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, qx, p.rows, width, qx_ld, many ? 128 : R);
    if (!mapped) return cudaErrorInvalidValue;
    if (many) return launch_many<T>(p, mw, mx, sms, st);
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
    if (!rows_apart(rows, outs, y_ld)) return fail(LSTM_ERR_INVALID, "bad argument: rows of an output overlap");
    if (outs > kMostColumns || width > kMostColumns) return fail(LSTM_ERR_UNSUPPORTED, "rows of more than 2^31 - 4096 columns");
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
