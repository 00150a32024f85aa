// 8-bit values (e4m3) with a scale for each 128 columns of a row, or for each 128 x 128 block: the largest magnitude of a block
// becomes 448, q = x / scale rounded to the nearest.  Bound by memory; every element is read once and stays in registers between
// the maximum and the rounding.  Rows: 25600 x 1312 of bf16 in 23.8 us, 0.66 of the copy rate, 73 % of the issue slots taken (17
// instructions an element: maxima, conversions, addresses; two of them, in pairs, make the quotient); blocks: 5000 x 6000 in 20 us, 0.69.
#include "../../include/lstm_b200.h"
#include "row_parts.cuh"

namespace lstm {
namespace {

struct QuantArgs {
    const void *x;
    long long x_ld;
    int rows, width;
    uint8_t *q;
    long long q_ld;
    float *scales;              // [ceil(rows / block rows)][ceil(width / 128)]
    int strips;                 // of a warp, where a scale belongs to one row
};

// A warp takes up to four neighbouring strips of one row (as many as divide the row evenly), all of them loaded first.
constexpr int kStripsPerWarp = 4;
template <typename T, int V>
__global__ void __launch_bounds__(256) fp8_quantize_rows_kernel(const __grid_constant__ QuantArgs p)
{
    const int lane = threadIdx.x & 31, blocks = (p.width + 127) / 128;
    const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (row >= p.rows) return;
    const int first = blockIdx.y * p.strips * kStrip;
    const T *from = (const T *)p.x + row * p.x_ld;
    Strip<T, V> raw[kStripsPerWarp];
#pragma unroll
    for (int j = 0; j < kStripsPerWarp; ++j)
        if (j < p.strips) raw[j].load(from, first + j * kStrip, p.width, lane);
#pragma unroll
    for (int j = 0; j < kStripsPerWarp; ++j) {
        const int c0 = first + j * kStrip;
        if (j >= p.strips || c0 >= p.width) break;
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = raw[j][i];
        unsigned top[2];
        strip_magnitudes<V>(x, lane, top);
        const float s0 = block_scale(top[0]), s1 = V == 8 ? s0 : block_scale(top[1]);
        const Units u0 = block_units(top[0], s0), u1 = V == 8 ? u0 : block_units(top[1], s1);
        store_strip_e4m3<V>(p.q + row * p.q_ld, c0, p.width, lane, x, u0, u1);
        float *out = p.scales + row * blocks + c0 / 128;
        if (lane == 0) out[0] = s0;
        if (lane == 16 && c0 + 128 < p.width) out[1] = s1;
    }
}

// A CTA takes 128 rows of one strip (two blocks), a warp ROWS of them: 8 in pairs of bf16, else 4, held as they were read, so that 32 warps
// fit an SM (one CTA of 16 warps with fp32 copies of 8 rows: 50 us for 5000 x 6000 of bf16).
template <typename T, int V, int ROWS>
__global__ void __launch_bounds__(128 / ROWS * 32, ROWS == 8 ? 2 : 1) fp8_quantize_blocks_kernel(const __grid_constant__ QuantArgs p)
{
    constexpr int kWarps = 128 / ROWS;
    __shared__ unsigned tops[kWarps][2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c0 = blockIdx.x * kStrip, blocks = (p.width + 127) / 128;
    const long long r0 = (long long)blockIdx.y * 128 + warp * ROWS;
    const int rows = (int)min((long long)ROWS, p.rows - r0);
    Strip<T, V> raw[ROWS];
    const T *from = (const T *)p.x + r0 * p.x_ld;
#pragma unroll
    for (int j = 0; j < ROWS; ++j)
        if (j < rows) raw[j].load(from + j * p.x_ld, c0, p.width, lane);
    unsigned top[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        if (j >= rows) break;
#pragma unroll
        for (int i = 0; i < 8; ++i) top[V == 8 ? 0 : i / 4] = max(top[V == 8 ? 0 : i / 4], magnitude(raw[j][i]));
    }
    if (V == 8) {                                       // lanes 0-15 hold the first block, 16-31 the second
#pragma unroll
        for (int o = 1; o < 16; o *= 2) top[0] = max(top[0], __shfl_xor_sync(0xffffffffu, top[0], o));
        top[1] = top[0];
    } else {
        top[0] = __reduce_max_sync(0xffffffffu, top[0]);
        top[1] = __reduce_max_sync(0xffffffffu, top[1]);
    }
    if (lane == 0) tops[warp][0] = top[0];
    if (lane == 16) tops[warp][1] = top[1];
    __syncthreads();
    top[0] = lane < kWarps ? tops[lane][0] : 0u;
    top[1] = lane < kWarps ? tops[lane][1] : 0u;
    top[0] = __reduce_max_sync(0xffffffffu, top[0]);
    top[1] = __reduce_max_sync(0xffffffffu, top[1]);
    const float s0 = block_scale(top[0]), s1 = block_scale(top[1]);
    const Units u0 = block_units(top[0], s0), u1 = block_units(top[1], s1), mine = V == 8 && lane >= 16 ? u1 : u0;
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        if (j >= rows) break;
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = raw[j][i];
        store_strip_e4m3<V>(p.q + (r0 + j) * p.q_ld, c0, p.width, lane, x, mine, u1);
    }
    if (threadIdx.x == 0) {
        float *out = p.scales + (long long)blockIdx.y * blocks + c0 / 128;
        out[0] = s0;
        if (c0 + 128 < p.width) out[1] = s1;
    }
}

template <typename T, int V>
void launch(QuantArgs &p, int block_rows, cudaStream_t st)
{
    constexpr int kRows = sizeof(T) * V == 2 || sizeof(T) == 4 ? 4 : 8;      // single bf16 take a register each, as fp32 do
    const int strips = (int)((p.width + (long long)kStrip - 1) / kStrip), groups = (strips + kStripsPerWarp - 1) / kStripsPerWarp;
    p.strips = (strips + groups - 1) / groups;
    if (block_rows == 1)
        fp8_quantize_rows_kernel<T, V><<<dim3((unsigned)((p.rows + 7ll) / 8), (unsigned)groups), 256, 0, st>>>(p);
    else
        fp8_quantize_blocks_kernel<T, V, kRows><<<dim3((unsigned)strips, (unsigned)((p.rows + 127ll) / 128)), 128 / kRows * 32, 0, st>>>(p);
}

template <typename T>
void by_vector(QuantArgs &p, int v, int block_rows, cudaStream_t st)
{
    if (v == 8) launch<T, 8>(p, block_rows, st);
    else if (v == 4) launch<T, 4>(p, block_rows, st);
    else if (v == 2) launch<T, 2>(p, block_rows, st);
    else launch<T, 1>(p, block_rows, st);
}

}  // namespace
}  // namespace lstm

using namespace lstm;

extern "C" int lstm_fp8_quantize(const void *x, long long x_ld, int rows, int width, int dtype, int block_rows, void *q, long long q_ld,
                                 float *scales, void *cuda_stream, char *err, int errlen)
{
    const Failure fail{err, errlen};
    if (rows < 0 || width < 1) return fail(LSTM_ERR_INVALID, "bad argument: rows must be 0 or more, width 1 or more");
    if (!known_type(dtype)) return fail(LSTM_ERR_INVALID, "bad argument: dtype must be LSTM_F32 or LSTM_BF16");
    if (block_rows != 1 && block_rows != 128) return fail(LSTM_ERR_INVALID, "bad argument: block_rows must be 1 or 128");
    if (rows == 0) return LSTM_OK;
    if (!x || !q || !scales) return fail(LSTM_ERR_INVALID, "bad argument: x, q and scales must be given");
    const int es = bytes_of(dtype);
    if (!aligned_to(x, es) || !aligned_to(scales, 4)) return fail(LSTM_ERR_INVALID, "bad argument: a pointer is not aligned to its elements");
    if (!aligned_to(q, 16) || q_ld % 16) return fail(LSTM_ERR_INVALID, "bad argument: 8-bit rows must start on 16 bytes");
    if (!rows_apart(rows, width, q_ld)) return fail(LSTM_ERR_INVALID, "bad argument: rows of an output overlap");
    if (block_rows == 128 && (rows + 127ll) / 128 > 65535) return fail(LSTM_ERR_UNSUPPORTED, "more than 65535 blocks of rows");
    if (width > kMostColumns) return fail(LSTM_ERR_UNSUPPORTED, "rows of more than 2^31 - 4096 columns");
    if (block_rows == 1 && (width + 1023ll) / 1024 > 65535) return fail(LSTM_ERR_UNSUPPORTED, "rows of more than 65535 x 1024 columns");
    int sms = 0;
    if (const int rc = device_sms(sms, fail)) return rc;
    RowAlignment al(width);
    al.matrix(x, x_ld, es);
    QuantArgs p = {x, x_ld, rows, width, (uint8_t *)q, q_ld, scales, 0};
    if (dtype == LSTM_BF16) by_vector<__nv_bfloat16>(p, al.v, block_rows, (cudaStream_t)cuda_stream);
    else by_vector<float>(p, al.v, block_rows, (cudaStream_t)cuda_stream);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? LSTM_OK : fail.cuda(e);
}
