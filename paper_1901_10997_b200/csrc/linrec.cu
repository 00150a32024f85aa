// Gated linear recurrence over whole sequences, forward and backward:
//
//     f_t = sigmoid(a_t), h_t = f_t h_{t-1} + (1 - f_t) x_t      (gate)      or     f_t = a_t, h_t = f_t h_{t-1} + x_t   (decay)
//
// The LSTM's cell with gates that do not see h_{t-1}: a step is the affine map h -> f h + b, maps compose to maps,
// (A2, H2) o (A1, H1) = (A2 A1, A2 H1 + H2), so spans of steps are reduced side by side and joined afterwards.
//
// A thread owns 16 consecutive steps of one vector of channels.  It loads them all at once (that is what keeps enough bytes
// in flight), reduces them to one map in registers, learns the state in front of its steps and runs through them once more
// from registers: inputs are read once and outputs written once.  Maps are joined in shared memory within a CTA and through
// distributed shared memory within a cluster of up to 16 CTAs that cover consecutive spans of time; one cluster barrier per
// 16 x CTAs x segments steps, no flags, no workspace, and an order of sums that does not depend on timing.
// State, maps and gates are fp32 throughout; outputs are rounded once.
//
// Backward: g_t = dh_t + f_{t+1} g_{t+1} is the same recurrence from the other end.  h is not read back: the forward pass
// leaves the fp32 state in front of every 16th step, and a thread recomputes its own 16 from there (1/4 byte an element
// instead of two for a rounded h, and h - x does not lose digits to that rounding).
#include "../../include/lstm_b200.h"
#include "operators.cuh"

namespace lstm {
namespace {

constexpr int kSeg = LSTM_LINREC_SEGMENT;   // steps per thread
constexpr int kThreads = 128;               // 3 to 4 CTAs an SM at 128 to 168 registers a thread

struct LinrecArgs {
    const void *a, *x;
    long long a_t, a_b, x_t, x_b;
    const float *h0;            // [B][D]; backward: dhT
    const int *lengths;
    int T, B, D, nvec;          // vectors of channels per sequence
    int gate, reverse, csize;
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

// f and 1 - f, both to full relative accuracy: with e = exp(-|u|) they are 1/(1+e) and e/(1+e), in the order that the sign says.
// bf16 data: the hardware's exponential (error 2^-22 and |u| 2^-24) is far inside a rounding to 8 bits; fp32 data: expf.
template <typename T>
__device__ __forceinline__ void gate_pair(float u, float &f, float &w)
{
    const float m = -fabsf(u);
    const float e = sizeof(T) == 2 ? ex2_fast(1.4426950408889634f * m) : expf(m);
    const float s = __fdividef(1.0f, 1.0f + e), r = e * s;
    f = u >= 0.0f ? s : r;
    w = u >= 0.0f ? r : s;
}

// h behind a map; a state of zero stays out of it, whatever the product of the decays grew to
__device__ __forceinline__ float apply_map(float A, float H, float h) { return h == 0.0f ? H : fmaf(A, h, H); }

template <int V>
struct alignas(8 * V) Map { float A[V], H[V]; };

template <int V>
__device__ __forceinline__ void join_behind(Map<V> &m, const Map<V> &later)      // m := later o m
{
#pragma unroll
    for (int v = 0; v < V; ++v) {
        m.H[v] = apply_map(later.A[v], later.H[v], m.H[v]);
        m.A[v] *= later.A[v];
    }
}

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// Shared by both directions: the joining of the threads' maps.
template <int V, int LX>
struct Joiner {
    static constexpr int kSegsPerWarp = 32 / LX;
    struct Shared {
        Map<V> warp[2][kThreads / 32][LX];
        Map<V> cta[2][16][LX];
    };
    // in: the thread's map and the carry in front of this span; out: the state in front of the thread, the carry behind the span
    static __device__ __forceinline__ void join(Shared &s, int parity, const Map<V> &mine, int csize, int rank, float (&carry)[V], float (&before)[V])
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = lane % LX, nwarps = blockDim.x >> 5;
        Map<V> m = mine;                // inclusive over the warp's segments
#pragma unroll
        for (int o = LX; o < 32; o *= 2) {
            Map<V> e;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                e.A[v] = __shfl_up_sync(0xffffffffu, m.A[v], o);
                e.H[v] = __shfl_up_sync(0xffffffffu, m.H[v], o);
            }
            if (lane >= o) {
                join_behind<V>(e, m);
                m = e;
            }
        }
        if (lane >= 32 - LX) s.warp[parity][warp][c] = m;
        Map<V> pre;                     // exclusive over the warp's segments
#pragma unroll
        for (int v = 0; v < V; ++v) { pre.A[v] = 1.0f; pre.H[v] = 0.0f; }
        if (LX < 32) {
            Map<V> e;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                e.A[v] = __shfl_up_sync(0xffffffffu, m.A[v], LX % 32);
                e.H[v] = __shfl_up_sync(0xffffffffu, m.H[v], LX % 32);
            }
            if (lane >= LX) pre = e;
        }
        __syncthreads();
        Map<V> front, all;              // of the CTA's warps: those in front of this one, all of them
#pragma unroll
        for (int v = 0; v < V; ++v) { all.A[v] = 1.0f; all.H[v] = 0.0f; }
        front = all;
        for (int w = 0; w < nwarps; ++w) {
            if (w == warp) front = all;
            join_behind<V>(all, s.warp[parity][w][c]);
        }
        float h[V];
        if (csize > 1) {
            if (threadIdx.x < LX) {
                const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(&s.cta[parity][rank][c]);
                for (int r = 0; r < csize; ++r) {
                    uint32_t there;
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine_at), "r"(r));
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there + 4 * v), "f"(all.A[v]) : "memory");
                        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there + 4 * (V + v)), "f"(all.H[v]) : "memory");
                    }
                }
            }
            cluster_arrive();
            cluster_wait();
#pragma unroll
            for (int v = 0; v < V; ++v) h[v] = carry[v];
            for (int r = 0; r < csize; ++r) {
                const Map<V> m2 = s.cta[parity][r][c];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    if (r == rank) h[v] = carry[v];
                    carry[v] = apply_map(m2.A[v], m2.H[v], carry[v]);
                }
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                h[v] = carry[v];
                carry[v] = apply_map(all.A[v], all.H[v], carry[v]);
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) before[v] = apply_map(pre.A[v], pre.H[v], apply_map(front.A[v], front.H[v], h[v]));
    }
};

template <typename T, int V, int LX>
__global__ void __launch_bounds__(kThreads, 4) linrec_forward_kernel(const __grid_constant__ LinrecArgs p)
{
    using J = Joiner<V, LX>;
    __shared__ typename J::Shared sh;
    const int rank = p.csize > 1 ? (int)cluster_rank() : 0;
    if (p.csize > 1) cluster_arrive();                  // the others' shared memory may be written once they have started
    const int c = threadIdx.x % LX, seg = threadIdx.x / LX, segs = blockDim.x / LX;
    const long long vec = (long long)(blockIdx.x / p.csize) * LX + c;
    const bool live = vec < (long long)p.B * p.nvec;
    const int b = live ? (int)(vec / p.nvec) : 0, d = live ? (int)(vec % p.nvec) * V : 0;
    int len = !live ? 0 : p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
    const int end = live ? p.T : 0;
    const long long bd = (long long)b * p.D + d, BD = (long long)p.B * p.D;
    float carry[V];
#pragma unroll
    for (int v = 0; v < V; ++v) carry[v] = live && p.h0 ? p.h0[bd + v] : 0.0f;
    const long long back = p.reverse ? -1 : 1;
    if (p.csize > 1) cluster_wait();

    const int span = kSeg * segs * p.csize;
    int parity = 0;
    for (long long base = 0; base < p.T; base += span, parity ^= 1) {
        const long long i0 = base + (long long)(rank * segs + seg) * kSeg;
        const long long t0 = p.reverse ? len - 1 - i0 : i0;
        const T *pa = (const T *)p.a + t0 * p.a_t + b * p.a_b + d, *px = (const T *)p.x + t0 * p.x_t + b * p.x_b + d;
        const long long sa = back * p.a_t, sx = back * p.x_t;
        const int n = (int)min((long long)kSeg, max(0ll, len - i0));
        float f[kSeg][V], add[kSeg][V];
        Vec<T, V> ra[kSeg], rx[kSeg];
#pragma unroll
        for (int k = 0; k < kSeg; ++k) {
            if (k < n) {
                ra[k] = load_vec<T, V>(pa + k * sa);
                rx[k] = load_vec<T, V>(px + k * sx);
            } else {
                ra[k] = rx[k] = zero_vec<T, V>();
            }
        }
        Map<V> m;
#pragma unroll
        for (int v = 0; v < V; ++v) { m.A[v] = 1.0f; m.H[v] = 0.0f; }
#pragma unroll
        for (int k = 0; k < kSeg; ++k) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float av = get<T, V>(ra[k], v), xv = get<T, V>(rx[k], v);
                float fv = av, bv = xv;
                if (p.gate) {
                    float w;
                    gate_pair<T>(av, fv, w);
                    bv = w * xv;
                }
                f[k][v] = k < n ? fv : 1.0f;
                add[k][v] = k < n ? bv : 0.0f;
                m.H[v] = fmaf(f[k][v], m.H[v], add[k][v]);
                m.A[v] *= f[k][v];
            }
        }
        float h[V];
        J::join(sh, parity, m, p.csize, rank, carry, h);
        if (p.states && i0 < end) store_vec<float, V>(p.states + (i0 / kSeg) * BD + bd, h);
        const int rows = (int)min((long long)kSeg, max(0ll, end - i0));
        T *ph = (T *)p.h + b * p.h_b + d;
#pragma unroll
        for (int k = 0; k < kSeg; ++k) {
            float o[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                h[v] = fmaf(f[k][v], h[v], add[k][v]);
                o[v] = k < n ? h[v] : 0.0f;
            }
            // steps behind a sequence's end lie at their own place in either direction
            if (k < rows) store_vec<T, V>(ph + (k < n ? t0 + back * k : i0 + k) * p.h_t, o);
        }
    }
    if (p.hT && live && rank == 0 && seg == 0) store_vec<float, V>(p.hT + bd, carry);
}

template <typename T, int V, int LX>
__global__ void __launch_bounds__(kThreads, 3) linrec_backward_kernel(const __grid_constant__ LinrecArgs p)
{
    using J = Joiner<V, LX>;
    __shared__ typename J::Shared sh;
    const int rank = p.csize > 1 ? (int)cluster_rank() : 0;
    if (p.csize > 1) cluster_arrive();
    const int c = threadIdx.x % LX, seg = threadIdx.x / LX, segs = blockDim.x / LX;
    const long long vec = (long long)(blockIdx.x / p.csize) * LX + c;
    const bool live = vec < (long long)p.B * p.nvec;
    const int b = live ? (int)(vec / p.nvec) : 0, d = live ? (int)(vec % p.nvec) * V : 0;
    const int len = !live ? 0 : p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
    const int end = live ? p.T : 0;
    const long long bd = (long long)b * p.D + d, BD = (long long)p.B * p.D;
    float carry[V];                                     // what reaches the state behind the steps that are left
#pragma unroll
    for (int v = 0; v < V; ++v) carry[v] = live && p.h0 ? p.h0[bd + v] : 0.0f;
    const long long back = p.reverse ? -1 : 1;
    if (p.csize > 1) cluster_wait();

    const long long nseg = (p.T + kSeg - 1) / kSeg;
    const int span = segs * p.csize;
    int parity = 0;
    for (long long base = 0; base < nseg; base += span, parity ^= 1) {
        const long long sg = nseg - 1 - (base + rank * segs + seg);
        const long long i0 = sg * kSeg;
        const long long t0 = p.reverse ? len - 1 - i0 : i0;
        const int n = sg < 0 ? 0 : (int)min((long long)kSeg, max(0ll, len - i0));
        const T *pa = (const T *)p.a + t0 * p.a_t + b * p.a_b + d, *px = (const T *)p.x + t0 * p.x_t + b * p.x_b + d;
        const T *pd = (const T *)p.dh + t0 * p.dh_t + b * p.dh_b + d;
        const long long sa = back * p.a_t, sx = back * p.x_t, sd = back * p.dh_t;
        Vec<T, V> ra[kSeg], rx[kSeg], rd[kSeg];
        float h[V];
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = 0.0f;
        if (n > 0) {
#pragma unroll
            for (int v = 0; v < V; ++v) h[v] = p.states[sg * BD + bd + v];
        }
#pragma unroll
        for (int k = 0; k < kSeg; ++k) {
            if (k < n) {
                ra[k] = load_vec<T, V>(pa + k * sa);
                rx[k] = load_vec<T, V>(px + k * sx);
                rd[k] = load_vec<T, V>(pd + k * sd);
            } else {
                ra[k] = rx[k] = rd[k] = zero_vec<T, V>();
            }
        }
        // da_t = g_t u_t and dx_t = g_t w_t with u = (h_{t-1} - x) f (1 - f), w = 1 - f  (decay: u = h_{t-1}, w = 1)
        float f[kSeg][V], u[kSeg][V], w[kSeg][V];
#pragma unroll
        for (int k = 0; k < kSeg; ++k) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float av = get<T, V>(ra[k], v), xv = get<T, V>(rx[k], v);
                float fv = av, wv = 1.0f, uv = h[v], bv = xv;
                if (p.gate) {
                    gate_pair<T>(av, fv, wv);
                    uv = (h[v] - xv) * (fv * wv);
                    bv = wv * xv;
                }
                h[v] = fmaf(fv, h[v], bv);
                f[k][v] = k < n ? fv : 1.0f;
                u[k][v] = uv;
                w[k][v] = wv;
            }
        }
        Map<V> m;
#pragma unroll
        for (int v = 0; v < V; ++v) { m.A[v] = 1.0f; m.H[v] = 0.0f; }
#pragma unroll
        for (int k = kSeg - 1; k >= 0; --k) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                m.H[v] = f[k][v] * (get<T, V>(rd[k], v) + m.H[v]);
                m.A[v] *= f[k][v];
            }
        }
        float q[V];
        J::join(sh, parity, m, p.csize, rank, carry, q);
        const int rows = sg < 0 ? 0 : (int)min((long long)kSeg, max(0ll, end - i0));
        T *pda = (T *)p.da + b * p.da_b + d, *pdx = (T *)p.h + b * p.h_b + d;
#pragma unroll
        for (int k = kSeg - 1; k >= 0; --k) {
            float oa[V], ox[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float g = get<T, V>(rd[k], v) + q[v];
                oa[v] = k < n ? g * u[k][v] : 0.0f;
                ox[v] = k < n ? g * w[k][v] : 0.0f;
                q[v] = f[k][v] * g;
            }
            if (k < rows) {
                const long long t = k < n ? t0 + back * k : i0 + k;
                store_vec<T, V>(pda + t * p.da_t, oa);
                store_vec<T, V>(pdx + t * p.h_t, ox);
            }
        }
    }
    if (p.hT && live && rank == 0 && seg == 0) store_vec<float, V>(p.hT + bd, carry);
}

template <typename T, int V, int LX>
cudaError_t launch(LinrecArgs &p, bool backward, int sms, cudaStream_t st)
{
    const void *fn = backward ? (const void *)linrec_backward_kernel<T, V, LX> : (const void *)linrec_forward_kernel<T, V, LX>;
    const long long groups = ((long long)p.B * p.nvec + LX - 1) / LX, need = ((long long)p.T + kSeg - 1) / kSeg;
    // segments of a CTA: whole warps, no more than there are steps for
    int segs = kThreads / LX;
    while (segs > 32 / LX && segs / 2 >= need) segs /= 2;
    // CTAs of a cluster: as many as leave no SM short of work, no more than there are steps for
    int csize = 1;
    while (csize < 16 && groups * csize < 4ll * sms && (long long)segs * csize < need) csize *= 2;
    p.csize = csize;
    if (groups * csize > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(groups * csize));
    cfg.blockDim = dim3((unsigned)(segs * LX));
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = csize;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = csize > 1 ? 1 : 0;
    if (csize > 8) {
        const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
    }
    void *args[] = {&p};
    return cudaLaunchKernelExC(&cfg, fn, args);
}

template <typename T, int V>
cudaError_t by_lanes(LinrecArgs &p, bool backward, int sms, cudaStream_t st)
{
    // 32 vectors side by side where there are channels enough for all SMs with clusters of 16, else 16 and two segments a warp
    const long long vecs = (long long)p.B * p.nvec;
    return vecs * 16 >= 32ll * 4 * sms || p.T <= 4 * kSeg ? launch<T, V, 32>(p, backward, sms, st) : launch<T, V, 16>(p, backward, sms, st);
}

template <typename T>
cudaError_t by_vector(LinrecArgs &p, bool backward, int sms, cudaStream_t st)
{
    const size_t es = sizeof(T);
    auto even = [&](const void *q, long long t, long long b) { return (uintptr_t)q % (2 * es) == 0 && t % 2 == 0 && b % 2 == 0; };
    auto even_f = [](const void *q) { return (uintptr_t)q % 8 == 0; };
    bool two = p.D % 2 == 0 && even(p.a, p.a_t, p.a_b) && even(p.x, p.x_t, p.x_b) && even(p.h, p.h_t, p.h_b) && even_f(p.hT) && even_f(p.states);
    if (backward) two = two && even(p.dh, p.dh_t, p.dh_b) && even(p.da, p.da_t, p.da_b);
    p.nvec = two ? p.D / 2 : p.D;
    return two ? by_lanes<T, 2>(p, backward, sms, st) : by_lanes<T, 1>(p, backward, sms, st);
}

int run(LinrecArgs &p, int dtype, bool backward, cudaStream_t st, const Failure &fail)
{
    int sms = 0;
    if (const int rc = device_sms(sms, fail)) return rc;
    const cudaError_t e = dtype == LSTM_BF16 ? by_vector<__nv_bfloat16>(p, backward, sms, st) : by_vector<float>(p, backward, sms, st);
    return e == cudaSuccess ? LSTM_OK : fail.cuda(e);
}

// what both calls refuse
int check(const void *a, const void *x, int T, int B, int D, int dtype, int flags, const Failure &fail)
{
    if (T < 0 || B < 0 || D < 1) return fail(LSTM_ERR_INVALID, "bad argument: T and B must be 0 or more, D 1 or more");
    if (!known_type(dtype)) return fail(LSTM_ERR_INVALID, "bad argument: dtype must be LSTM_F32 or LSTM_BF16");
    if (flags & ~(LSTM_LINREC_GATE | LSTM_LINREC_REVERSE)) return fail(LSTM_ERR_INVALID, "bad argument: unknown flags");
    if (T > 0 && B > 0 && (!a || !x)) return fail(LSTM_ERR_INVALID, "bad argument: a and x must be given");
    return LSTM_OK;
}

bool aligned(const void *p, int dtype) { return aligned_to(p, bytes_of(dtype)); }

}  // namespace
}  // namespace lstm

using namespace lstm;

extern "C" {

int lstm_linear_recurrence(const void *a, long long a_t, long long a_b, const void *x, long long x_t, long long x_b, const float *h0,
                           const int *lengths, int T, int B, int D, int dtype, int flags, void *h, long long h_t, long long h_b, float *hT,
                           float *states, void *cuda_stream, char *err, int errlen)
{
    const Failure fail{err, errlen};
    if (const int rc = check(a, x, T, B, D, dtype, flags, fail)) return rc;
    if (T > 0 && B > 0 && !h) return fail(LSTM_ERR_INVALID, "bad argument: h must be given");
    if (!aligned(a, dtype) || !aligned(x, dtype) || !aligned(h, dtype) || !aligned(h0, LSTM_F32) || !aligned(hT, LSTM_F32) ||
        !aligned(states, LSTM_F32) || !aligned(lengths, LSTM_F32))
        return fail(LSTM_ERR_INVALID, "bad argument: a pointer is not aligned to its elements");
    if (B == 0 || (T == 0 && !hT)) return LSTM_OK;
    LinrecArgs p = {};
    p.a = a; p.a_t = a_t; p.a_b = a_b;
    p.x = x; p.x_t = x_t; p.x_b = x_b;
    p.h0 = h0; p.lengths = lengths;
    p.T = T; p.B = B; p.D = D;
    p.gate = flags & LSTM_LINREC_GATE ? 1 : 0;
    p.reverse = flags & LSTM_LINREC_REVERSE ? 1 : 0;
    p.h = h; p.h_t = h_t; p.h_b = h_b;
    p.hT = hT; p.states = states;
    return run(p, dtype, false, (cudaStream_t)cuda_stream, fail);
}

int lstm_linear_recurrence_backward(const void *a, long long a_t, long long a_b, const void *x, long long x_t, long long x_b,
                                    const float *states, const void *dh, long long dh_t, long long dh_b, const float *dhT,
                                    const int *lengths, int T, int B, int D, int dtype, int flags, void *da, long long da_t, long long da_b,
                                    void *dx, long long dx_t, long long dx_b, float *dh0, void *cuda_stream, char *err, int errlen)
{
    const Failure fail{err, errlen};
    if (const int rc = check(a, x, T, B, D, dtype, flags, fail)) return rc;
    if (T > 0 && B > 0 && (!states || !dh || !da || !dx)) return fail(LSTM_ERR_INVALID, "bad argument: states, dh, da and dx must be given");
    if (!aligned(a, dtype) || !aligned(x, dtype) || !aligned(dh, dtype) || !aligned(da, dtype) || !aligned(dx, dtype) ||
        !aligned(states, LSTM_F32) || !aligned(dhT, LSTM_F32) || !aligned(dh0, LSTM_F32) || !aligned(lengths, LSTM_F32))
        return fail(LSTM_ERR_INVALID, "bad argument: a pointer is not aligned to its elements");
    if (B == 0 || (T == 0 && !dh0)) return LSTM_OK;
    LinrecArgs p = {};
    p.a = a; p.a_t = a_t; p.a_b = a_b;
    p.x = x; p.x_t = x_t; p.x_b = x_b;
    p.h0 = dhT; p.lengths = lengths;
    p.T = T; p.B = B; p.D = D;
    p.gate = flags & LSTM_LINREC_GATE ? 1 : 0;
    p.reverse = flags & LSTM_LINREC_REVERSE ? 1 : 0;
    p.h = dx; p.h_t = dx_t; p.h_b = dx_b;
    p.hT = dh0; p.states = const_cast<float *>(states);
    p.dh = dh; p.dh_t = dh_t; p.dh_b = dh_b;
    p.da = da; p.da_t = da_t; p.da_b = da_b;
    return run(p, dtype, true, (cudaStream_t)cuda_stream, fail);
}

}  // extern "C"
