// Root-mean-square norm of rows, with the residual's addition in front and 8-bit values with scales behind where wanted:
//
//     r = x + residual        y = r rstd w        rstd = 1 / sqrt(mean(r^2) + eps)
//
// and its gradients  dx = rstd (w dy - r rstd^2 mean(w dy r)) + dr,   dw = sum over rows of dy r rstd.
//
// Bound by memory: a row is read once into the registers of one warp (up to 512 columns) or of up to 16, summed by shuffles, and
// written once.  Sums are fp32 over at most 32 elements a lane before they are joined pairwise.
// Share of the copy rate, bf16: 25600 x 1500 with residual 0.98 (48 us), 25600 x 1600 to 8 bits 0.81 (54 us: 72 % of the issue slots taken),
// gradients of 25600 x 1500 0.80 (58 us); rows that start anywhere (odd widths) are read two bytes at a time: 0.73, 0.56 and 0.43.
#include "../../include/lstm_b200.h"
#include "row_parts.cuh"

namespace lstm {
namespace {

struct NormArgs {
    const void *x, *residual;
    long long x_ld, residual_ld;
    const float *w;
    float eps;
    int rows, width;
    void *y;
    long long y_ld;
    float *scales;              // not NULL: y is e4m3
    void *r;
    long long r_ld;
    float each;                 // 1 / width
};

// 1 / sqrt(v): the hardware's approximation and one Newton step; 0 gives infinity, infinity 0
__device__ __forceinline__ float reciprocal_root(float v)
{
    const float y = rsqrtf(v), better = fmaf(0.5f * y, fmaf(-v * y, y, 1.0f), y);
    return v > 0.0f && v < __int_as_float(0x7f800000) ? better : y;
}

// NS strips a warp.  Up to two strips, a warp has a row to itself and four stand in a CTA; wider rows have a CTA each, whose
// warps meet once.  Few registers a thread and many CTAs: that, not the work of a thread, is what keeps the memory busy.
constexpr int kNormWarps = 16;
template <typename T, int V, int NS, bool ALONE>
__global__ void __launch_bounds__(ALONE ? 128 : 512, ALONE ? 12 : NS == 2 ? 2 : 1) rms_norm_kernel(const __grid_constant__ NormArgs p)
{
    __shared__ float s[kNormWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int first = ALONE ? 0 : warp, warps = ALONE ? 1 : blockDim.x >> 5;
    const long long row = ALONE ? (long long)blockIdx.x * 4 + warp : blockIdx.x;
    if (row >= p.rows) return;                          // whole warps where they do not meet
    const T *x = (const T *)p.x + row * p.x_ld, *res = p.residual ? (const T *)p.residual + row * p.residual_ld : nullptr;
    float r[NS][8];
    {
        Strip<T, V> a[NS], b[NS];
#pragma unroll
        for (int j = 0; j < NS; ++j) a[j].load(x, (first + j * warps) * kStrip, p.width, lane);
        if (res) {
#pragma unroll
            for (int j = 0; j < NS; ++j) b[j].load(res, (first + j * warps) * kStrip, p.width, lane);
        }
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) r[j][i] = a[j][i];
        if (res) {
#pragma unroll
            for (int j = 0; j < NS; ++j) {
                float add[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) add[i] = b[j][i];
                add_vec<8>(r[j], r[j], add);
            }
        }
    }
    float part[8] = {};
#pragma unroll
    for (int j = 0; j < NS; ++j) fma_vec<8>(part, r[j], r[j], part);
    float sum = ((part[0] + part[1]) + (part[2] + part[3])) + ((part[4] + part[5]) + (part[6] + part[7]));
#pragma unroll
    for (int o = 16; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (!ALONE) {
        if (lane == 0) s[warp] = sum;
        __syncthreads();
        sum = 0.0f;
        for (int i = 0; i < warps; ++i) sum += s[i];
    }
    const float rstd = reciprocal_root(sum * p.each + p.eps);
    float rs[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rs[i] = rstd;
#pragma unroll
    for (int j = 0; j < NS; ++j) {
        const int c0 = (first + j * warps) * kStrip;
        if (c0 >= p.width) break;
        // the norm continues from the sum as it is, not from the rounded copy that is handed on: one rounding an output
        if (p.r) store_strip<T, V>((T *)p.r + row * p.r_ld, c0, p.width, lane, r[j]);
        float w[8], y[8];
        load_strip<float, V>(p.w, c0, p.width, lane, w);
        mul_vec<8>(y, r[j], rs);
        mul_vec<8>(y, y, w);
        if (!p.scales) {
            store_strip<T, V>((T *)p.y + row * p.y_ld, c0, p.width, lane, y);
            continue;
        }
        unsigned top[2];
        strip_magnitudes<V>(y, lane, top);
        const float s0 = block_scale(top[0]), s1 = V == 8 ? s0 : block_scale(top[1]);
        const Units u0 = block_units(top[0], s0), u1 = V == 8 ? u0 : block_units(top[1], s1);
        store_strip_e4m3<V>((uint8_t *)p.y + row * p.y_ld, c0, p.width, lane, y, u0, u1);
        const int blocks = (p.width + 127) / 128;
        float *out = p.scales + row * blocks + c0 / 128;
        if (lane == 0) out[0] = s0;
        if (lane == 16 && c0 + 128 < p.width) out[1] = s1;
    }
}

struct NormBackArgs {
    const void *dy, *r, *dr;
    long long dy_ld, r_ld, dr_ld;
    const float *w;
    float eps;
    int rows, width;
    void *dx;
    long long dx_ld;
    float *part;                // [CTAs][width] partial sums of dw
};

// A CTA walks over rows, NS strips a warp; a thread keeps its columns of dw from row to row.  With one or two strips it keeps those of
// w too and has the next row's loads under way while it works on one (25600 x 1500 without: 148 us); four leave no registers for it.
constexpr int kBackWarps = 16;
template <typename T, int V, int NS, bool DR>
struct BackRow {
    Strip<T, V> r[NS], dy[NS], dr[DR ? NS : 1];
    __device__ __forceinline__ void load(const NormBackArgs &p, long long row, int first, int warps, int lane)
    {
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            const int c0 = (first + j * warps) * kStrip;
            r[j].load((const T *)p.r + row * p.r_ld, c0, p.width, lane);
            dy[j].load((const T *)p.dy + row * p.dy_ld, c0, p.width, lane);
            if (DR && p.dr) dr[DR ? j : 0].load((const T *)p.dr + row * p.dr_ld, c0, p.width, lane);
        }
    }
};

template <typename T, int V, int NS>
__global__ void __launch_bounds__(NS == 4 ? 512 : 256) rms_norm_backward_kernel(const __grid_constant__ NormBackArgs p)
{
    constexpr bool kAhead = NS <= 2;
    __shared__ float2 s[2][kBackWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    float w[kAhead ? NS : 1][8], dw[NS][8];
#pragma unroll
    for (int j = 0; j < NS; ++j) {
        if (kAhead) load_strip<float, V>(p.w, (warp + j * warps) * kStrip, p.width, lane, w[kAhead ? j : 0]);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[j][i] = 0.0f;
    }
    typedef BackRow<T, V, NS, kAhead> Row;
    Row now, next;
    long long row = blockIdx.x;
    if (kAhead && row < p.rows) next.load(p, row, warp, warps, lane);
    const float each = 1.0f / (float)p.width;
    for (int turn = 0; row < p.rows; row += gridDim.x, turn ^= 1) {
        if (kAhead) {
            now = next;
            if (row + gridDim.x < p.rows) next.load(p, row + gridDim.x, warp, warps, lane);
        } else {
            now.load(p, row, warp, warps, lane);
        }
        float rr = 0.0f, ry = 0.0f;
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            if (!kAhead) load_strip<float, V>(p.w, (warp + j * warps) * kStrip, p.width, lane, w[0]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float r = now.r[j][i];
                rr = fmaf(r, r, rr);
                ry = fmaf(r, w[kAhead ? j : 0][i] * now.dy[j][i], ry);
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o /= 2) {
            rr += __shfl_xor_sync(0xffffffffu, rr, o);
            ry += __shfl_xor_sync(0xffffffffu, ry, o);
        }
        if (warps > 1) {
            if (lane == 0) s[turn][warp] = make_float2(rr, ry);
            __syncthreads();                            // the other set is read no more once all have come here
            rr = ry = 0.0f;
            for (int i = 0; i < warps; ++i) { rr += s[turn][i].x; ry += s[turn][i].y; }
        }
        const float rstd = reciprocal_root(rr * each + p.eps);
        const float mean = ry * each * rstd * rstd;
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            const int c0 = (warp + j * warps) * kStrip;
            if (!kAhead) {
                load_strip<float, V>(p.w, c0, p.width, lane, w[0]);
                if (p.dr) now.dr[0].load((const T *)p.dr + row * p.dr_ld, c0, p.width, lane);
            }
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float r = now.r[j][i], dy = now.dy[j][i];
                dw[j][i] = fmaf(dy, r * rstd, dw[j][i]);
                o[i] = rstd * (w[kAhead ? j : 0][i] * dy - r * mean);
                if (p.dr) o[i] += now.dr[kAhead ? j : 0][i];
            }
            store_strip<T, V>((T *)p.dx + row * p.dx_ld, c0, p.width, lane, o);
        }
    }
#pragma unroll
    for (int j = 0; j < NS; ++j)
        store_strip<float, V>(p.part + (long long)blockIdx.x * p.width, (warp + j * warps) * kStrip, p.width, lane, dw[j]);
}

// dw = sum of the CTAs' rows, always in the same order: 32 columns a CTA, thread (column, i) adds rows i, i + 32, ...
__global__ void __launch_bounds__(1024) rms_norm_join_kernel(const float *part, int parts, int width, float *dw)
{
    __shared__ float s[32][33];
    const int c = blockIdx.x * 32 + threadIdx.x;
    float sum = 0.0f;
    if (c < width) {
#pragma unroll 8
        for (int i = threadIdx.y; i < parts; i += 32) sum += part[(long long)i * width + c];
    }
    s[threadIdx.y][threadIdx.x] = sum;
    __syncthreads();
    float v = s[threadIdx.x][threadIdx.y];
#pragma unroll
    for (int o = 16; o > 0; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    const int col = blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x == 0 && col < width) dw[col] = v;
}

// strips of a warp and warps of a CTA for a width: few strips a warp, and no idle one but in the last
struct RowShape {
    int ns, warps;
    RowShape(int width, bool backward)
    {
        const int strips = (width + kStrip - 1) / kStrip;
        ns = strips <= (backward ? 16 : 32) ? 2 : 4;
        warps = (strips + ns - 1) / ns;
    }
};
template <typename T, int V>
void launch_norm(const NormArgs &p, cudaStream_t st)
{
    const RowShape s(p.width, false);
    if (s.warps == 1) rms_norm_kernel<T, V, 2, true><<<(unsigned)((p.rows + 3ll) / 4), 128, 0, st>>>(p);
    else if (s.ns == 2) rms_norm_kernel<T, V, 2, false><<<p.rows, s.warps * 32, 0, st>>>(p);
    else rms_norm_kernel<T, V, 4, false><<<p.rows, s.warps * 32, 0, st>>>(p);
}

// the most CTAs of the backward kernel, each of which leaves a row of partial sums: 16 warps an SM
int parts_of(int rows, int width, int sms)
{
    const RowShape s(width, true);
    const int resident = s.warps >= 16 ? 1 : 16 / s.warps;
    return rows < sms * resident ? rows : sms * resident;
}
// ... of which as many are launched as are resident at once; returns how many
template <typename T, int V, int NS>
int launch_back_shape(const NormBackArgs &p, int warps, int parts, int sms, cudaStream_t st)
{
    static std::atomic<int> resident[kBackWarps + 1];
    int n = resident[warps].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, rms_norm_backward_kernel<T, V, NS>, warps * 32, 0) != cudaSuccess || n < 1) n = 1;
        resident[warps].store(n, std::memory_order_relaxed);
    }
    if (parts > n * sms) parts = n * sms;
    rms_norm_backward_kernel<T, V, NS><<<parts, warps * 32, 0, st>>>(p);
    return parts;
}
template <typename T, int V>
int launch_back(const NormBackArgs &p, int parts, int sms, cudaStream_t st)
{
    const RowShape s(p.width, true);
    return s.ns == 2 ? launch_back_shape<T, V, 2>(p, s.warps, parts, sms, st) : launch_back_shape<T, V, 4>(p, s.warps, parts, sms, st);
}

template <template <typename, int> class F, typename... A>
void by_type(int dtype, int v, A &&...a)
{
    const bool half = dtype == LSTM_BF16;
    if (v == 8) half ? F<__nv_bfloat16, 8>::go(a...) : F<float, 8>::go(a...);
    else if (v == 4) half ? F<__nv_bfloat16, 4>::go(a...) : F<float, 4>::go(a...);
    else if (v == 2) half ? F<__nv_bfloat16, 2>::go(a...) : F<float, 2>::go(a...);
    else half ? F<__nv_bfloat16, 1>::go(a...) : F<float, 1>::go(a...);
}
template <typename T, int V> struct Forward { static void go(const NormArgs &p, cudaStream_t st) { launch_norm<T, V>(p, st); } };
template <typename T, int V> struct Backward { static void go(const NormBackArgs &p, int &parts, int sms, cudaStream_t st) { parts = launch_back<T, V>(p, parts, sms, st); } };

int check(int rows, int width, int dtype, float eps, const Failure &fail)
{
    if (rows < 0 || width < 1) return fail(LSTM_ERR_INVALID, "bad argument: rows must be 0 or more, width 1 or more");
    if (width > LSTM_RMS_NORM_MAX_WIDTH) return fail(LSTM_ERR_UNSUPPORTED, "rows of more than LSTM_RMS_NORM_MAX_WIDTH columns are not served");
    if (!known_type(dtype)) return fail(LSTM_ERR_INVALID, "bad argument: dtype must be LSTM_F32 or LSTM_BF16");
    if (!(eps >= 0.0f)) return fail(LSTM_ERR_INVALID, "bad argument: eps must be 0 or more");
    return LSTM_OK;
}

}  // namespace
}  // namespace lstm

using namespace lstm;

extern "C" {

int lstm_rms_norm(const void *x, long long x_ld, const void *residual, long long residual_ld, const float *w, float eps, int rows, int width,
                  int dtype, void *y, long long y_ld, float *scales, void *r, long long r_ld, void *cuda_stream, char *err, int errlen)
{
    const Failure fail{err, errlen};
    if (const int rc = check(rows, width, dtype, eps, fail)) return rc;
    if (rows == 0) return LSTM_OK;
    if (!x || !w || !y) return fail(LSTM_ERR_INVALID, "bad argument: x, w and y must be given");
    const int es = bytes_of(dtype);
    if (!aligned_to(x, es) || !aligned_to(residual, es) || !aligned_to(r, es) || !aligned_to(w, 4) || !aligned_to(scales, 4) || (!scales && !aligned_to(y, es)))
        return fail(LSTM_ERR_INVALID, "bad argument: a pointer is not aligned to its elements");
    if (scales && (!aligned_to(y, 16) || y_ld % 16))
        return fail(LSTM_ERR_INVALID, "bad argument: 8-bit rows must start on 16 bytes");
    if (!rows_apart(rows, width, y_ld) || (r && !rows_apart(rows, width, r_ld))) return fail(LSTM_ERR_INVALID, "bad argument: rows of an output overlap");
    int sms = 0;
    if (const int rc = device_sms(sms, fail)) return rc;
    RowAlignment al(width);
    al.matrix(x, x_ld, es);
    al.matrix(residual, residual_ld, es);
    al.matrix(r, r_ld, es);
    al.matrix(w, 0, 4);
    if (!scales) al.matrix(y, y_ld, es);
    NormArgs p = {x, residual, x_ld, residual_ld, w, eps, rows, width, y, y_ld, scales, r, r_ld, 1.0f / (float)width};
    by_type<Forward>(dtype, al.v, p, (cudaStream_t)cuda_stream);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? LSTM_OK : fail.cuda(e);
}

int lstm_rms_norm_backward(const void *dy, long long dy_ld, const void *r, long long r_ld, const float *w, const void *dr, long long dr_ld,
                           float eps, int rows, int width, int dtype, void *dx, long long dx_ld, float *dw, float *workspace,
                           long long workspace_floats, void *cuda_stream, char *err, int errlen)
{
    const Failure fail{err, errlen};
    if (const int rc = check(rows, width, dtype, eps, fail)) return rc;
    if (!dw) return fail(LSTM_ERR_INVALID, "bad argument: dw must be given");
    if (rows > 0 && (!dy || !r || !w || !dx)) return fail(LSTM_ERR_INVALID, "bad argument: dy, r, w and dx must be given");
    const int es = bytes_of(dtype);
    if (!aligned_to(dy, es) || !aligned_to(r, es) || !aligned_to(dr, es) || !aligned_to(dx, es) || !aligned_to(w, 4) || !aligned_to(dw, 4) ||
        !aligned_to(workspace, 4))
        return fail(LSTM_ERR_INVALID, "bad argument: a pointer is not aligned to its elements");
    if (!rows_apart(rows, width, dx_ld)) return fail(LSTM_ERR_INVALID, "bad argument: rows of an output overlap");
    int sms = 0;
    if (const int rc = device_sms(sms, fail)) return rc;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    int parts = parts_of(rows, width, sms);
    if (parts > 0 && (!workspace || workspace_floats < (long long)parts * width))
        return fail(LSTM_ERR_INVALID, "bad argument: the workspace is smaller than lstm_rms_norm_workspace says");
    if (parts > 0) {
        RowAlignment al(width);
        al.matrix(dy, dy_ld, es);
        al.matrix(r, r_ld, es);
        al.matrix(dr, dr_ld, es);
        al.matrix(dx, dx_ld, es);
        al.matrix(w, 0, 4);
        al.matrix(workspace, 0, 4);
        NormBackArgs p = {dy, r, dr, dy_ld, r_ld, dr_ld, w, eps, rows, width, dx, dx_ld, workspace};
        by_type<Backward>(dtype, al.v, p, parts, sms, st);
    }
    rms_norm_join_kernel<<<(width + 31) / 32, dim3(32, 32), 0, st>>>(workspace, parts, width, dw);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? LSTM_OK : fail.cuda(e);
}

long long lstm_rms_norm_workspace(int rows, int width)
{
    int sms = 0;
    if (rows < 0 || width < 1 || width > LSTM_RMS_NORM_MAX_WIDTH || device_sms(sms, Failure{nullptr, 0}) != LSTM_OK) return -1;
    return (long long)parts_of(rows, width, sms) * width;
}

}  // extern "C"
