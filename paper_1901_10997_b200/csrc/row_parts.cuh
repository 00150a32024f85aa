// Rows of a matrix in the registers of a warp: the unit is a strip of 256 columns, 8 elements a lane, of which lane l holds
// 8 / V vectors of V neighbours (vector q: columns q * 32 V + l V).  V follows the alignment of the rows, so that every access of a
// warp is one run of memory whatever it is; a block of 128 columns lies in one warp for every V.
#pragma once
#include "operators.cuh"

#include <cuda_fp8.h>

namespace lstm {

constexpr int kStrip = 256;
constexpr float kE4m3Max = 448.0f;

template <int V>
__device__ __forceinline__ int strip_col(int q, int lane) { return q * 32 * V + lane * V; }

// lane's 8 elements of the strip at column c0; columns behind `width` read as zero
// (whole strips without a question for each vector: their addresses are one register and constants)
// as they lie in memory, so that a row's loads can all be under way before the first is looked at
template <typename T, int V>
struct Strip {
    Vec<T, V> v[8 / V];
    __device__ __forceinline__ void load(const T *row, int c0, int width, int lane)
    {
        const T *at = row + c0 + lane * V;
        if (c0 + kStrip <= width) {
#pragma unroll
            for (int q = 0; q < 8 / V; ++q) v[q] = load_vec<T, V>(at + q * 32 * V);
        } else {
#pragma unroll
            for (int q = 0; q < 8 / V; ++q) v[q] = c0 + strip_col<V>(q, lane) < width ? load_vec<T, V>(at + q * 32 * V) : zero_vec<T, V>();
        }
    }
    __device__ __forceinline__ float operator[](int i) const { return get<T, V>(v[i / V], i % V); }
};
template <typename T, int V>
__device__ __forceinline__ void load_strip(const T *row, int c0, int width, int lane, float (&o)[8])
{
    Strip<T, V> s;
    s.load(row, c0, width, lane);
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = s[i];
}
template <typename T, int V>
__device__ __forceinline__ void store_strip(T *row, int c0, int width, int lane, const float (&o)[8])
{
    T *at = row + c0 + lane * V;
    if (c0 + kStrip <= width) {
#pragma unroll
        for (int q = 0; q < 8 / V; ++q) store_raw<T, V>(at + q * 32 * V, to_vec<T, V>(&o[q * V]));
    } else {
#pragma unroll
        for (int q = 0; q < 8 / V; ++q)
            if (c0 + strip_col<V>(q, lane) < width) store_raw<T, V>(at + q * 32 * V, to_vec<T, V>(&o[q * V]));
    }
}

// |x| as an integer of the same order, in which NaN is above infinity
__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// What becomes 448: the largest magnitude of a block, at least 448 * 2^-126 (blocks of zeros, and those whose scale would be subnormal).
__device__ __forceinline__ float block_top(unsigned largest) { return __uint_as_float(max(largest, 0x04e00000u)); }
// The scale of a block: a normal number, so that its reciprocal is finite; a block that holds an infinity or NaN gets that as its scale.
__device__ __forceinline__ float block_scale(unsigned largest)
{
    const float top = block_top(largest), t = top * (1.0f / kE4m3Max);
    const float s = fmaf(fmaf(-t, kE4m3Max, top), 1.0f / kE4m3Max, t);       // corrected by its remainder
    return largest < 0x7f800000u ? s : top;
}
// What an element is multiplied by to be in units of the unrounded scale: 448 / max |x| = hi + lo to some 45 bits, so that x hi + x lo is rounded
// once and a quotient that e4m3 holds, or that is a tie of it, comes out exactly.  Few digits make ties: by the rounded scale, one in twenty thousand
// bf16 values fell on the wrong side of its tie; by its reciprocal alone one in some ten thousand of any.
// (Beside an infinite value finite ones are zero.)
struct Units { float hi, lo; };
__device__ __forceinline__ Units block_units(unsigned largest, float scale)
{
    float hi;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(hi) : "f"(scale));
    const float lo = fmaf(-hi, block_top(largest), kE4m3Max) * (hi * (1.0f / kE4m3Max));
    return {hi, largest < 0x7f800000u ? lo : 0.0f};
}
__device__ __forceinline__ void in_units(float (&y)[4], const float (&x)[4], Units u)
{
    const float hi[4] = {u.hi, u.hi, u.hi, u.hi}, lo[4] = {u.lo, u.lo, u.lo, u.lo};
    float t[4];
    mul_vec<4>(t, x, lo);
    fma_vec<4>(y, x, hi, t);
}
// two values as e4m3, the nearest, at most 448 in magnitude
__device__ __forceinline__ unsigned to_e4m3x2(float a, float b)
{
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

// largest magnitude of the lane's elements in block `half` of the strip, over the lanes that share the block
template <int V>
__device__ __forceinline__ void strip_magnitudes(const float (&y)[8], int lane, unsigned (&top)[2])
{
    top[0] = top[1] = 0u;
    if (V == 8) {                                       // a lane is in one block: lanes 0-15 the first, 16-31 the second
#pragma unroll
        for (int i = 0; i < 8; ++i) top[0] = max(top[0], magnitude(y[i]));
#pragma unroll
        for (int o = 1; o < 16; o *= 2) top[0] = max(top[0], __shfl_xor_sync(0xffffffffu, top[0], o));
        top[1] = top[0];                                // each lane's own block in both places
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            top[0] = max(top[0], magnitude(y[i]));
            top[1] = max(top[1], magnitude(y[4 + i]));
        }
        top[0] = __reduce_max_sync(0xffffffffu, top[0]);
        top[1] = __reduce_max_sync(0xffffffffu, top[1]);
    }
}

// the lane's 8 elements, in units of their blocks' scales, as e4m3 bytes
template <int V>
__device__ __forceinline__ void store_strip_e4m3(uint8_t *row, int c0, int width, int lane, const float (&x)[8], Units u0, Units u1)
{
    const bool whole = c0 + kStrip <= width;
    const float lo[4] = {x[0], x[1], x[2], x[3]}, hi[4] = {x[4], x[5], x[6], x[7]};
    float a[4], b[4];
    in_units(a, lo, u0);
    in_units(b, hi, V == 8 ? u0 : u1);
    const float y[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
#pragma unroll
    for (int q = 0; q < 8 / V; ++q) {
        const int c = c0 + strip_col<V>(q, lane);
        if (!whole && c >= width) continue;
        unsigned w[V == 8 ? 2 : 1];
        if (V == 1) {
            w[0] = to_e4m3x2(y[q], 0.0f);
            row[c] = (uint8_t)w[0];
        } else if (V == 2) {
            w[0] = to_e4m3x2(y[2 * q], y[2 * q + 1]);
            *reinterpret_cast<unsigned short *>(row + c) = (unsigned short)w[0];
        } else {
#pragma unroll
            for (int i = 0; i < V / 4; ++i)
                w[i] = to_e4m3x2(y[q * V + 4 * i], y[q * V + 4 * i + 1]) | to_e4m3x2(y[q * V + 4 * i + 2], y[q * V + 4 * i + 3]) << 16;
            if (V == 4) *reinterpret_cast<unsigned *>(row + c) = w[0];
            if (V == 8) *reinterpret_cast<uint2 *>(row + c) = make_uint2(w[0], w[V == 8 ? 1 : 0]);
        }
    }
}

// widest vector (8, 4, 2 or 1 elements) that divides the width and to which every matrix's rows are aligned
struct RowAlignment {
    int v;
    explicit RowAlignment(int width) : v(8) { while (width % v) v /= 2; }
    void matrix(const void *p, long long ld, int bytes)
    {
        if (!p) return;
        auto fits = [&](int n) { const int word = n * bytes < 16 ? n * bytes : 16; return (uintptr_t)p % word == 0 && ld * bytes % word == 0; };
        while (v > 1 && !fits(v)) v /= 2;
    }
};

}  // namespace lstm
