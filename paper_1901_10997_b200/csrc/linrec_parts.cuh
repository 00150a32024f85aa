// What the kernels of the gated linear recurrence (linrec.cu, linrec_wide.cu) share: arguments, gates, maps, inputs fetched ahead.
#pragma once
#include "operators.cuh"

namespace lstm {

struct LinrecArgs {
    const void *a, *x;
    long long a_t, a_b, x_t, x_b;
    const float *h0;            // [B][D]; backward: dhT
    const int *lengths;
    int T, B, D, nvec;          // vectors of channels per sequence
    int gate, reverse, csize;
    int chunks, chunk_len;      // time cut into chunks that run side by side (linrec_wide.cu): T = chunks * chunk_len or less
    float *maps;                // [2][chunks][B][D] and the initial carries [B][D], where there is more than one
    void *h;                    // backward: dx
    long long h_t, h_b;
    float *hT;                  // [B][D]; backward: dh0
    float *states;              // [ceil(T/16)][B][D]
    // backward
    const void *dh;
    long long dh_t, dh_b;
    void *da;
    long long da_t, da_b;
};

__device__ __forceinline__ float rcp_fast(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// f and 1 - f, both to full relative accuracy: with e = exp(-|u|) they are 1/(1+e) and e/(1+e), in the order that the sign says.
// bf16 data: the hardware's exponential (error 2^-22 and |u| 2^-24) is far inside a rounding to 8 bits; fp32 data: expf.
// u -> f and w = 1 - f
template <typename T, int V>
__device__ __forceinline__ void gate_vec(const float (&u)[V], float (&f)[V], float (&w)[V])
{
    float e[V], s[V], r[V], one[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        e[v] = sizeof(T) == 2 ? ex2_fast(-1.4426950408889634f * fabsf(u[v])) : expf(-fabsf(u[v]));
        one[v] = 1.0f;
    }
    add_vec<V>(s, e, one);
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = rcp_fast(s[v]);
    mul_vec<V>(r, e, s);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const bool open = u[v] >= 0.0f;
        f[v] = open ? s[v] : r[v];
        w[v] = open ? r[v] : s[v];
    }
}

template <int V>
struct alignas(8 * V) Map { float A[V], H[V]; };

template <int V>
__device__ __forceinline__ Map<V> identity()
{
    Map<V> m;
#pragma unroll
    for (int v = 0; v < V; ++v) { m.A[v] = 1.0f; m.H[v] = 0.0f; }
    return m;
}
template <int V>
__device__ __forceinline__ void apply(const Map<V> &m, float (&h)[V])
{
    fma_vec<V>(h, m.A, h, m.H);
}
// m := later o m.  A product of decays that grew out of range is held at its edge: a state of zero stays zero behind it.  A NaN stays
// (fminf and fmaxf would take the edge in its place).
__device__ __forceinline__ float within(float x, float edge)
{
    float y;
    asm("{\n\t.reg .f32 e;\n\tneg.f32 e, %2;\n\tmin.NaN.f32 %0, %1, %2;\n\tmax.NaN.f32 %0, %0, e;\n\t}" : "=f"(y) : "f"(x), "f"(edge));
    return y;
}
template <int V, bool GATE>
__device__ __forceinline__ float held(float A) { return GATE ? A : within(A, 3.4028235e38f); }
// What a span's first step adds, from which its H starts.  A decay that is NaN or infinite makes it NaN: the state behind such a step is not
// finite, whatever was in front of it, and by A alone, which is held, it could become so again.
template <int V, bool GATE>
__device__ __forceinline__ void first_added(float (&H)[V], const float (&f)[V], const float (&add)[V])
{
    const float zero[V] = {};
    if (GATE) {
#pragma unroll
        for (int v = 0; v < V; ++v) H[v] = add[v];
    } else {
        fma_vec<V>(H, f, zero, add);
    }
}
template <int V, bool GATE>
__device__ __forceinline__ void join_behind(Map<V> &m, const Map<V> &later)
{
    apply<V>(later, m.H);
#pragma unroll
    for (int v = 0; v < V; ++v) m.A[v] = held<V, GATE>(m.A[v] * later.A[v]);
}

// what stands in the place of a step's logit or decay to keep the state
template <typename T, int V, bool GATE>
__device__ __forceinline__ Vec<T, V> keep()
{
    float o[V];
#pragma unroll
    for (int v = 0; v < V; ++v) o[v] = GATE ? __int_as_float(0x7f800000) : 1.0f;
    return to_vec<T, V>(o);
}

// ---------------------------------------------------------------------------------------------------
// A thread's inputs, DEPTH spans ahead of their use: N matrices, STEPS vectors of each, in a CTA of THREADS.
// InShared: asynchronous copies of 4, 8 or 16 bytes into places of the thread's own in shared memory (nobody else touches them: no
// barrier).  InRegisters: one span ahead, for vectors of two bytes, which such a copy does not have, and where registers serve better.
// ---------------------------------------------------------------------------------------------------
template <typename T, int V, int N, bool GATE, int STEPS, int THREADS, int DEPTH>
struct InShared {
    static constexpr int kSteps = STEPS, kThreads = THREADS, kBytes = sizeof(T) * V, kDepth = DEPTH;
    static constexpr int kSmem = (kDepth + 1) * N * kSteps * kThreads * kBytes;
    unsigned char *mine;
    int put = 0, take = 0;
    __device__ explicit InShared(unsigned char *smem) : mine(smem + threadIdx.x * kBytes) {}
    static __device__ __forceinline__ int place(int stage, int i, int k) { return ((stage * N + i) * kSteps + k) * kThreads * kBytes; }
    // n steps of N matrices, from p[i] on, step[i] elements apart
    __device__ __forceinline__ void fetch(const T *const (&p)[N], const long long (&step)[N], int n)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t to = smem_u32(mine + place(put, i, 0));
            const T *q = p[i];
            if (n == kSteps) {
#pragma unroll
                for (int k = 0; k < kSteps; ++k) {
                    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to + k * kThreads * kBytes), "l"(q), "n"(kBytes) : "memory");
                    q += step[i];
                }
            } else {                    // steps behind the end keep the state
                for (int k = 0; k < kSteps; ++k) {
                    if (k < n) asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to + k * kThreads * kBytes), "l"(q), "n"(kBytes) : "memory");
                    else *reinterpret_cast<Vec<T, V> *>(mine + place(put, i, k)) = i == 0 ? keep<T, V, GATE>() : zero_vec<T, V>();
                    q += step[i];
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        put = put == kDepth ? 0 : put + 1;
    }
    __device__ __forceinline__ void arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(kDepth) : "memory"); }
    __device__ __forceinline__ Vec<T, V> get_vec(int i, int k) const { return *reinterpret_cast<const Vec<T, V> *>(mine + place(take, i, k)); }
    __device__ __forceinline__ void next_if_registers() {}
    __device__ __forceinline__ void next() { take = take == kDepth ? 0 : take + 1; }
};
template <typename T, int V, int N, bool GATE, int STEPS>
struct InRegisters {
    static constexpr int kSteps = STEPS, kDepth = 1, kSmem = 0;
    Vec<T, V> held[2][N][kSteps];
    __device__ explicit InRegisters(unsigned char *) {}
    __device__ __forceinline__ void fetch(const T *const (&p)[N], const long long (&step)[N], int n)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const T *q = p[i];
            if (n == kSteps) {
#pragma unroll
                for (int k = 0; k < kSteps; ++k) { held[1][i][k] = load_vec<T, V>(q); q += step[i]; }
            } else {
#pragma unroll
                for (int k = 0; k < kSteps; ++k) {
                    held[1][i][k] = k < n ? load_vec<T, V>(q) : i == 0 ? keep<T, V, GATE>() : zero_vec<T, V>();
                    q += step[i];
                }
            }
        }
    }
    __device__ __forceinline__ void arrived() {}
    __device__ __forceinline__ Vec<T, V> get_vec(int i, int k) const { return held[0][i][k]; }
    __device__ __forceinline__ void next() {}
    __device__ __forceinline__ void next_if_registers()
    {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int k = 0; k < kSteps; ++k) held[0][i][k] = held[1][i][k];
    }
};

// steps of a span of STEPS from i0 that lie in front of `last`
template <int STEPS>
__device__ __forceinline__ int count_steps(long long i0, int last)
{
    return i0 < 0 || i0 >= last ? 0 : min(STEPS, last - (int)i0);
}

// The kernels for many channels, and for chunks of time (linrec_wide.cu); a vector has v channels.
// How many chunks a call is cut into, and their length (a multiple of 64): the same for a call's workspace and its launch.
int linrec_chunks(int T, int B, int D, int &chunk_len);
bool linrec_wide_serves(const LinrecArgs &p, int v, bool bf16, bool backward, int sms, int &wide_v);
cudaError_t launch_linrec_wide(LinrecArgs &p, int v, bool bf16, bool backward, cudaStream_t st);

}  // namespace lstm
