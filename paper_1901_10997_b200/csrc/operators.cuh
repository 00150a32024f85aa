// What the stateless operators (linrec.cu, rms_norm.cu, fp8_quantize.cu, fp8_product.cu) share: failures at the C boundary,
// the device's SM count, vectors of elements.
#pragma once
#include "device_util.cuh"

#include <atomic>
#include <cstdio>

namespace lstm {

// the reason of a failure, in the caller's buffer (which may be missing)
struct Failure {
    char *err;
    int errlen;
    int operator()(int code, const char *why) const
    {
        if (err && errlen > 0) snprintf(err, (size_t)errlen, "%s", why);
        return code;
    }
    // a failed CUDA call; its error is not left behind for the next caller to find
    int cuda(cudaError_t e) const
    {
        (void)cudaGetLastError();
        return (*this)(LSTM_ERR_CUDA, cudaGetErrorString(e));
    }
};

// SMs of the current device, which must run sm_100a code
inline int device_sms(int &sms, const Failure &fail)
{
    static std::atomic<int> known[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return fail.cuda(e);
    if (dev >= 0 && dev < 64 && (sms = known[dev].load(std::memory_order_relaxed)) > 0) return LSTM_OK;
    int major = 0;
    if ((e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev)) != cudaSuccess) return fail.cuda(e);
    if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return fail.cuda(e);
    if (major != 10) return fail(LSTM_ERR_CUDA, "the current device does not run sm_100a code");
    if (dev >= 0 && dev < 64) known[dev].store(sms, std::memory_order_relaxed);
    return LSTM_OK;
}

// The attributes that a kernel needs once on each device; `done` is the kernel's own, a bit for each device.
inline cudaError_t prepare_kernel(const void *fn, std::atomic<unsigned long long> &done, int dynamic_smem, bool large_clusters)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
    if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, dynamic_smem);
    if (e == cudaSuccess && large_clusters) e = cudaFuncSetAttribute(fn, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
    return e;
}

// ---------------------------------------------------------------------------------------------------
// V elements of type T (float or __nv_bfloat16), loaded and stored as one word of up to 16 bytes
// ---------------------------------------------------------------------------------------------------
template <int BYTES> struct WordOf;
template <> struct WordOf<2> { typedef unsigned short type; };
template <> struct WordOf<4> { typedef unsigned type; };
template <> struct WordOf<8> { typedef uint2 type; };
template <> struct WordOf<16> { typedef uint4 type; };

// Kept as the words that were loaded: two bf16 in a register stay one until they are looked at.
template <typename T, int V>
struct alignas(sizeof(T) * V <= 16 ? sizeof(T) * V : 16) Vec {
    static constexpr int kBytes = sizeof(T) * V, kHeld = kBytes < 4 ? 1 : kBytes / 4;
    typedef typename WordOf<kBytes < 4 ? kBytes : 4>::type Held;
    Held w[kHeld];
};

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load_vec(const T *p)
{
    constexpr int kBytes = sizeof(T) * V, kWord = kBytes <= 16 ? kBytes : 16;
    typedef typename WordOf<kWord>::type W;
    union { Vec<T, V> v; W w[kBytes / kWord]; } u;
#pragma unroll
    for (int i = 0; i < kBytes / kWord; ++i) u.w[i] = reinterpret_cast<const W *>(p)[i];
    return u.v;
}
template <typename T, int V>
__device__ __forceinline__ Vec<T, V> zero_vec()
{
    Vec<T, V> v;
#pragma unroll
    for (int i = 0; i < Vec<T, V>::kHeld; ++i) v.w[i] = 0;
    return v;
}
template <typename T, int V>
__device__ __forceinline__ float get(const Vec<T, V> &v, int i)
{
    if (sizeof(T) == 4) return __uint_as_float(v.w[i]);
    const unsigned pair = v.w[i / 2];
    return __uint_as_float(i % 2 ? pair & 0xffff0000u : pair << 16);
}
// rounds to nearest, ties to even
template <typename T, int V>
__device__ __forceinline__ Vec<T, V> to_vec(const float *o)
{
    Vec<T, V> v;
    if (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < Vec<T, V>::kHeld; ++i) v.w[i] = __float_as_uint(o[i]);
    } else if (V == 1) {
        v.w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(o[0]));
    } else {
#pragma unroll
        for (int i = 0; i + 1 < V; i += 2) {
            const __nv_bfloat162 pair = __floats2bfloat162_rn(o[i], o[i + 1]);
            v.w[i / 2] = *reinterpret_cast<const unsigned *>(&pair);
        }
    }
    return v;
}
template <typename T, int V>
__device__ __forceinline__ void store_raw(T *p, const Vec<T, V> &v)
{
    constexpr int kBytes = sizeof(T) * V, kWord = kBytes <= 16 ? kBytes : 16;
    typedef typename WordOf<kWord>::type W;
    union { Vec<T, V> v; W w[kBytes / kWord]; } u;
    u.v = v;
#pragma unroll
    for (int i = 0; i < kBytes / kWord; ++i) reinterpret_cast<W *>(p)[i] = u.w[i];
}
template <typename T, int V>
__device__ __forceinline__ void store_vec(T *p, const float (&o)[V]) { store_raw<T, V>(p, to_vec<T, V>(o)); }

// ---------------------------------------------------------------------------------------------------
// fp32 arithmetic on V values, two to an instruction: d = a b + c, d = a b, d = a + b
// ---------------------------------------------------------------------------------------------------
template <int V>
__device__ __forceinline__ void fma_vec(float (&d)[V], const float (&a)[V], const float (&b)[V], const float (&c)[V])
{
    if (V == 1) { d[0] = fmaf(a[0], b[0], c[0]); return; }
#pragma unroll
    for (int v = 0; v + 1 < V; v += 2)
        asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
            "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
            : "=f"(d[v]), "=f"(d[v + 1]) : "f"(a[v]), "f"(a[v + 1]), "f"(b[v]), "f"(b[v + 1]), "f"(c[v]), "f"(c[v + 1]));
}
template <int V>
__device__ __forceinline__ void mul_vec(float (&d)[V], const float (&a)[V], const float (&b)[V])
{
    if (V == 1) { d[0] = a[0] * b[0]; return; }
#pragma unroll
    for (int v = 0; v + 1 < V; v += 2)
        asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
            : "=f"(d[v]), "=f"(d[v + 1]) : "f"(a[v]), "f"(a[v + 1]), "f"(b[v]), "f"(b[v + 1]));
}
template <int V>
__device__ __forceinline__ void add_vec(float (&d)[V], const float (&a)[V], const float (&b)[V])
{
    if (V == 1) { d[0] = a[0] + b[0]; return; }
#pragma unroll
    for (int v = 0; v + 1 < V; v += 2)
        asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
            : "=f"(d[v]), "=f"(d[v + 1]) : "f"(a[v]), "f"(a[v + 1]), "f"(b[v]), "f"(b[v + 1]));
}

// rows of an output share no element
inline bool rows_apart(int rows, int width, long long ld) { return rows < 2 || ld >= width || ld <= -(long long)width; }
// ... nor do the runs of D elements of an output [T][B][D]: none begins within another
inline bool steps_apart(int T, int B, int D, long long t, long long b)
{
    t = t < 0 ? -t : t;
    b = b < 0 ? -b : b;
    if (T < 2 || B < 2) return (T < 2 || t >= D) && (B < 2 || b >= D);
    if (t < D || b < D) return false;
    if (t < b) { const long long s = t; t = b; b = s; const int n = T; T = B; B = n; }
    if ((t - D) / b >= B - 1) return true;              // the inner ones all lie between two of the outer
    for (long long j = 1; j < B; ++j)                   // strides that cross (of either sign): is j b within D of a multiple of t?
        for (long long i = j * b / t; i <= j * b / t + 1 && i < T; ++i) {
            const long long off = j * b - i * t;
            if (off < D && off > -D) return false;
        }
    return true;
}

constexpr int kMostColumns = 0x7ffff000;                 // of a row: the end of its last strip, block or tile is still counted in 32 bits
inline bool known_type(int dtype) { return dtype == LSTM_F32 || dtype == LSTM_BF16; }
inline int bytes_of(int dtype) { return dtype == LSTM_BF16 ? 2 : 4; }
inline bool aligned_to(const void *p, int bytes) { return (uintptr_t)p % (unsigned)bytes == 0; }

}  // namespace lstm
