// Gated linear recurrence over whole sequences, forward and backward:
//
//     f_t = sigmoid(a_t), h_t = f_t h_{t-1} + (1 - f_t) x_t      (gate)      or     f_t = a_t, h_t = f_t h_{t-1} + x_t   (decay)
//
// The LSTM's cell with gates that do not see h_{t-1}: a step is the affine map h -> f h + b, maps compose to maps,
// (A2, H2) o (A1, H1) = (A2 A1, A2 H1 + H2), so spans of steps are reduced side by side and joined afterwards.
//
// The kernels here serve calls with few channels (linrec_wide.cu has those for many channels, for long sequences in chunks of time and
// for a few steps; linrec_wide_serves says which).  A thread owns 8 or 16 consecutive steps of a vector of up to four channels.  It reduces them to one map in registers, learns the
// state in front of its steps and runs through them once more from registers: inputs are read once and outputs written once.
// Maps are joined by shuffles within a warp, in shared memory within a CTA and through distributed shared memory within a cluster
// whose CTAs cover consecutive spans of time: no flags in global memory, no workspace, and an order of sums that does not
// depend on timing.  Inputs come two spans ahead of their use by asynchronous copies into places of the thread's own in shared
// memory, so that neither the joining nor a barrier holds them up.
// What bounds them is the length of the chain of joinings (about 2 us a round of 128 steps a CTA): 200 x 8 x 700 of bf16 takes 6 us, 4096 x
// 1500 20, where their bytes take 1 and 6.
// State, maps and gates are fp32 throughout; outputs are rounded once.
//
// Backward: g_t = dh_t + f_{t+1} g_{t+1} is the same recurrence from the other end.  h is not read back: the forward pass
// leaves the fp32 state in front of every 16th step, and its steps are run through again from there (1/4 byte an element
// instead of two for a rounded h, and h - x does not lose digits to that rounding).
#include "../../include/lstm_b200.h"
#include "linrec_parts.cuh"

#include <type_traits>

namespace lstm {
namespace {

constexpr int kThreads = 128;
constexpr int kMaxCluster = 16;

// How a warp's lanes are laid out for vectors of V channels: 32 channels side by side, and V spans of time.
template <int V>
struct Lay {
    static constexpr int kLanes = 32 / V;                   // vectors side by side
    static constexpr int kSpans = V;                        // spans of a warp, one behind the other
    static constexpr int kSteps = V == 1 ? 16 : 8;          // steps of a span
    static constexpr int kWarpSteps = kSpans * kSteps;      // a multiple of the 16 steps between saved states
    static_assert(kWarpSteps % LSTM_LINREC_SEGMENT == 0 && LSTM_LINREC_SEGMENT == 16, "a warp begins at a saved state");
};

__device__ __forceinline__ uint32_t cluster_rank()
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
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// V floats to another CTA's shared memory, counted by its barrier
template <int V>
__device__ __forceinline__ void send(uint32_t to, const float (&v)[V], uint32_t bar)
{
    if (V == 4)
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                     ::"r"(to), "f"(v[0]), "f"(v[V > 1 ? 1 : 0]), "f"(v[V > 2 ? 2 : 0]), "f"(v[V > 3 ? 3 : 0]), "r"(bar) : "memory");
    else if (V == 2)
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];"
                     ::"r"(to), "f"(v[0]), "f"(v[V > 1 ? 1 : 0]), "r"(bar) : "memory");
    else
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.f32 [%0], %1, [%2];" ::"r"(to), "f"(v[0]), "r"(bar) : "memory");
}

// ---------------------------------------------------------------------------------------------------
// The joining of the threads' maps, the same in both directions.  Every thread holds the carry of its channels: the state in front
// of the spans that the cluster is working on.  `order` counts a warp's spans in the order in which they are joined.
// ---------------------------------------------------------------------------------------------------
template <int V, bool GATE>
struct Joiner {
    typedef Lay<V> L;
    struct Shared {
        Map<V> warp[2][kThreads / 32][L::kLanes];
        Map<V> cta[2][kMaxCluster][L::kLanes];
        alignas(8) unsigned long long bar[2];
        int gave_up;
    };
    Shared &s;
    const int csize, rank, c, order, warp, nwarps;
    int turn = 0;               // joinings so far; the two sets of shared memory are used in turn

    __device__ Joiner(Shared &s_, int csize_)
        : s(s_), csize(csize_), rank(csize_ > 1 ? (int)cluster_rank() : 0), c(threadIdx.x % L::kLanes), order(threadIdx.x % 32 / L::kLanes),
          warp(threadIdx.x / 32), nwarps(blockDim.x / 32)
    {
        if (csize == 1) return;
        if (threadIdx.x == 0) {
            s.gave_up = 0;
            mbar_init(smem_u32(&s.bar[0]), 1);
            mbar_init(smem_u32(&s.bar[1]), 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        cluster_arrive();       // waited for in ready(): the others' barriers stand before anything is sent to them
    }
    __device__ void ready() const { if (csize > 1) cluster_wait(); }
    __device__ void leave() const
    {
        if (csize > 1) { cluster_arrive(); cluster_wait(); }
    }

    // mine: the thread's map; carry: in front of these spans -> behind them; before: the state in front of the thread's steps
    __device__ __forceinline__ void join(const Map<V> &mine, float (&carry)[V], float (&before)[V])
    {
        const int set = turn & 1;
        Map<V> upto = mine;             // the warp's spans up to this one
#pragma unroll
        for (int o = 1; o < L::kSpans; o *= 2) {
            Map<V> e;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                e.A[v] = __shfl_up_sync(0xffffffffu, upto.A[v], o * L::kLanes);
                e.H[v] = __shfl_up_sync(0xffffffffu, upto.H[v], o * L::kLanes);
            }
            if (order >= o) {
                join_behind<V, GATE>(e, upto);
                upto = e;
            }
        }
        if (order == L::kSpans - 1) s.warp[set][warp][c] = upto;
        __syncthreads();
        float h[V];
        if (csize > 1) {
            const uint32_t bar = smem_u32(&s.bar[set]);
            if (warp == 0) {            // the CTA's map goes to all CTAs of the cluster
                if (threadIdx.x == 0) mbar_expect_tx(bar, csize * L::kLanes * (int)sizeof(Map<V>));
                Map<V> all = s.warp[set][0][c];
                for (int w = 1; w < nwarps; ++w) join_behind<V, GATE>(all, s.warp[set][w][c]);
                const uint32_t slot = smem_u32(&s.cta[set][rank][c]);
                for (int r = order; r < csize; r += L::kSpans) {
                    const uint32_t to = at_rank(slot, r), their = at_rank(bar, r);
                    send<V>(to, all.A, their);
                    send<V>(to + 4 * V, all.H, their);
                }
            }
            // a set is written again two joinings on, by CTAs that have this CTA's map of the one between, which is sent
            // when all of its threads have read this one
            const bool ok = mbar_wait(bar, (turn >> 1) & 1, &s.gave_up);
            for (int r = 0; r < rank; ++r) apply<V>(s.cta[set][r][c], carry);
#pragma unroll
            for (int v = 0; v < V; ++v) h[v] = carry[v];
            for (int r = rank; r < csize; ++r) apply<V>(s.cta[set][r][c], carry);
            if (!ok) {                  // a wait that gave up leaves NaN, not something that looks like a result
#pragma unroll
                for (int v = 0; v < V; ++v) h[v] = carry[v] = __uint_as_float(0x7fffffffu);
            }
            for (int w = 0; w < warp; ++w) apply<V>(s.warp[set][w][c], h);
        } else {
            for (int w = 0; w < warp; ++w) apply<V>(s.warp[set][w][c], carry);
#pragma unroll
            for (int v = 0; v < V; ++v) h[v] = carry[v];
            for (int w = warp; w < nwarps; ++w) apply<V>(s.warp[set][w][c], carry);
        }
        ++turn;
        if (L::kSpans > 1) {
            Map<V> e;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                e.A[v] = __shfl_up_sync(0xffffffffu, upto.A[v], L::kLanes % 32);
                e.H[v] = __shfl_up_sync(0xffffffffu, upto.H[v], L::kLanes % 32);
            }
            if (order > 0) apply<V>(e, h);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) before[v] = h[v];
    }
};

// the values have been loaded when a thread gets past here
template <int V>
__device__ __forceinline__ void arrived(float (&v)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) asm volatile("mov.f32 %0, %0;" : "+f"(v[i])::"memory");
}

// What a thread works on
template <int V>
struct Place {
    int b, d, len, end;         // steps of the sequence; of the batch (0 where there is no such channel)
    long long bd, BD;
    bool live;
    __device__ explicit Place(const LinrecArgs &p)
    {
        const long long vec = (long long)(blockIdx.x / p.csize) * Lay<V>::kLanes + threadIdx.x % Lay<V>::kLanes;
        live = vec < (long long)p.B * p.nvec;
        b = live ? (int)(vec / p.nvec) : 0;
        d = live ? (int)(vec % p.nvec) * V : 0;
        len = !live ? 0 : p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
        end = live ? p.T : 0;
        bd = (long long)b * p.D + d;
        BD = (long long)p.B * p.D;
    }
    static __device__ __forceinline__ int count(long long i0, int last) { return count_steps<Lay<V>::kSteps>(i0, last); }
};

// vectors of two bytes wait in registers, the others two spans ahead in shared memory
template <typename T, int V, int N, bool GATE>
using Ahead = std::conditional_t<sizeof(T) * V == 2, InRegisters<T, V, N, GATE, Lay<V>::kSteps>, InShared<T, V, N, GATE, Lay<V>::kSteps, kThreads, 2>>;

template <typename T, int V, bool GATE>
__global__ void __launch_bounds__(kThreads, 4) linrec_forward_kernel(const __grid_constant__ LinrecArgs p)
{
    typedef Lay<V> L;
    constexpr int kSteps = L::kSteps;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ typename Joiner<V, GATE>::Shared sh;
    Joiner<V, GATE> joiner(sh, p.csize);
    const Place<V> at(p);
    const long long sign = p.reverse ? -1 : 1;
    const long long step[2] = {sign * p.a_t, sign * p.x_t}, out_step = sign * p.h_t;
    T *ph = (T *)p.h + at.b * p.h_b + at.d;

    const int span = blockDim.x / L::kLanes * p.csize * kSteps;
    long long i0 = (long long)(joiner.rank * (blockDim.x / L::kLanes) + threadIdx.x / L::kLanes) * kSteps;
    Ahead<T, V, 2, GATE> in(smem);
    const T *from[2];
    {
        const long long t0 = p.reverse ? at.len - 1 - i0 : i0;
        from[0] = (const T *)p.a + at.b * p.a_b + at.d + t0 * p.a_t;
        from[1] = (const T *)p.x + at.b * p.x_b + at.d + t0 * p.x_t;
    }
    const long long jump[2] = {span * step[0], span * step[1]};
    long long ahead = i0;
    auto fetch = [&]() {
        in.fetch(from, step, Place<V>::count(ahead, at.len));
        ahead += span;
        from[0] += jump[0];
        from[1] += jump[1];
    };
#pragma unroll
    for (int i = 0; i < Ahead<T, V, 2, GATE>::kDepth; ++i) fetch();
    float carry[V];
#pragma unroll
    for (int v = 0; v < V; ++v) carry[v] = at.live && p.h0 ? p.h0[at.bd + v] : 0.0f;
    arrived<V>(carry);                  // another thread may write the final state over it
    joiner.ready();
    for (long long base = 0; base < p.T; base += span, i0 += span) {
        const int n = Place<V>::count(i0, at.len);
        in.next_if_registers();
        fetch();
        in.arrived();
        const bool idle = __all_sync(0xffffffffu, n == 0);      // behind the end of all its sequences a warp only joins in
        float f[kSteps][V], add[kSteps][V];
        Map<V> m = identity<V>();
        if (!idle) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const Vec<T, V> ra = in.get_vec(0, k), rx = in.get_vec(1, k);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                f[k][v] = get<T, V>(ra, v);
                add[k][v] = get<T, V>(rx, v);
            }
            if (GATE) {
                float w[V];
                gate_vec<T, V>(f[k], f[k], w);
                mul_vec<V>(add[k], add[k], w);
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) m.A[v] = f[0][v];
        first_added<V, GATE>(m.H, f[0], add[0]);
#pragma unroll
        for (int k = 1; k < kSteps; ++k) {
            fma_vec<V>(m.H, f[k], m.H, add[k]);
            mul_vec<V>(m.A, m.A, f[k]);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) m.A[v] = held<V, GATE>(m.A[v]);
        }
        in.next();
        float h[V];
        joiner.join(m, carry, h);
        if (p.states && i0 < at.end && i0 % LSTM_LINREC_SEGMENT == 0)
            store_vec<float, V>(p.states + i0 / LSTM_LINREC_SEGMENT * at.BD + at.bd, h);
        const long long t0 = p.reverse ? at.len - 1 - i0 : i0;
        if (n == kSteps) {
            T *q = ph + t0 * p.h_t;
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                fma_vec<V>(h, f[k], h, add[k]);
                store_vec<T, V>(q, h);
                q += out_step;
            }
        } else if (idle) {
            const float zero[V] = {};
            const int rows = Place<V>::count(i0, at.end);
            for (int k = 0; k < rows; ++k) store_vec<T, V>(ph + (i0 + k) * p.h_t, zero);
        } else {
            const int rows = Place<V>::count(i0, at.end);
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                float o[V];
                fma_vec<V>(h, f[k], h, add[k]);
#pragma unroll
                for (int v = 0; v < V; ++v) o[v] = k < n ? h[v] : 0.0f;
                // steps behind a sequence's end lie at their own place in either direction
                if (k < rows) store_vec<T, V>(ph + (k < n ? (p.reverse ? t0 - k : t0 + k) : i0 + k) * p.h_t, o);
            }
        }
    }
    if (p.hT && at.live && joiner.rank == 0 && threadIdx.x < L::kLanes) store_vec<float, V>(p.hT + at.bd, carry);
    joiner.leave();
}

template <typename T, int V, bool GATE>
__global__ void __launch_bounds__(kThreads, V == 4 ? 2 : 3) linrec_backward_kernel(const __grid_constant__ LinrecArgs p)
{
    typedef Lay<V> L;
    constexpr int kSteps = L::kSteps;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ typename Joiner<V, GATE>::Shared sh;
    Joiner<V, GATE> joiner(sh, p.csize);
    const Place<V> at(p);
    const long long sign = p.reverse ? -1 : 1;
    const long long step[3] = {sign * p.a_t, sign * p.x_t, sign * p.dh_t};
    T *pda = (T *)p.da + at.b * p.da_b + at.d, *pdx = (T *)p.h + at.b * p.h_b + at.d;

    // Spans are joined from the last to the first: the first in the joining are the latest in the order of processing.
    const long long nspan = ((long long)p.T + L::kWarpSteps - 1) / L::kWarpSteps * L::kSpans;
    const int span = blockDim.x / L::kLanes * p.csize * kSteps;
    long long i0 = (nspan - 1 - (long long)(joiner.rank * (blockDim.x / L::kLanes) + threadIdx.x / L::kLanes)) * kSteps;
    const bool begins = i0 % LSTM_LINREC_SEGMENT == 0;      // a saved state stands in front of the thread's steps
    Ahead<T, V, 3, GATE> in(smem);
    const T *from[3];
    {
        const long long t0 = p.reverse ? at.len - 1 - i0 : i0;
        from[0] = (const T *)p.a + at.b * p.a_b + at.d + t0 * p.a_t;
        from[1] = (const T *)p.x + at.b * p.x_b + at.d + t0 * p.x_t;
        from[2] = (const T *)p.dh + at.b * p.dh_b + at.d + t0 * p.dh_t;
    }
    long long ahead = i0;
    const long long jump[3] = {span * step[0], span * step[1], span * step[2]};
    auto fetch = [&]() {
        in.fetch(from, step, Place<V>::count(ahead, at.len));
        ahead -= span;
#pragma unroll
        for (int i = 0; i < 3; ++i) from[i] -= jump[i];
    };
    auto saved = [&](long long i, float (&h)[V]) {
        const bool here = begins && i >= 0 && i < at.len;
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = here ? p.states[i / LSTM_LINREC_SEGMENT * at.BD + at.bd + v] : 0.0f;
    };
#pragma unroll
    for (int i = 0; i < Ahead<T, V, 3, GATE>::kDepth; ++i) fetch();
    float carry[V], hs[V];                              // carry: what reaches the state behind the steps that are left
#pragma unroll
    for (int v = 0; v < V; ++v) carry[v] = at.live && p.h0 ? p.h0[at.bd + v] : 0.0f;
    saved(i0, hs);
    arrived<V>(carry);
    joiner.ready();
    for (long long base = 0; base < nspan * kSteps; base += span, i0 -= span) {
        const int n = Place<V>::count(i0, at.len);
        in.next_if_registers();
        fetch();
        in.arrived();
        // da_t = g_t u_t and dx_t = g_t w_t with u = (h_{t-1} - x) f (1 - f), w = 1 - f  (decay: u = h_{t-1}, w = 1)
        const bool idle = __all_sync(0xffffffffu, n == 0);
        float f[kSteps][V], u[kSteps][V], w[kSteps][V], d[kSteps][V];
        Map<V> m = identity<V>();
        if (!idle) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const Vec<T, V> ra = in.get_vec(0, k), rx = in.get_vec(1, k), rd = in.get_vec(2, k);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                f[k][v] = get<T, V>(ra, v);
                u[k][v] = get<T, V>(rx, v);
                d[k][v] = get<T, V>(rd, v);
                w[k][v] = 1.0f;
            }
            if (GATE) gate_vec<T, V>(f[k], f[k], w[k]);
        }
        float h[V];
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = hs[v];
        if (V > 1) {
            // the state behind the first 8 of a segment's steps is the one in front of its other 8, which the lanes below hold
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                float b[V];
                mul_vec<V>(b, w[k], u[k]);
                fma_vec<V>(h, f[k], h, b);
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float behind = __shfl_down_sync(0xffffffffu, h[v], L::kLanes % 32);
                h[v] = begins ? hs[v] : behind;
            }
        }
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            float b[V], fw[V], less[V];
            if (GATE) {
#pragma unroll
                for (int v = 0; v < V; ++v) less[v] = h[v] - u[k][v];
                mul_vec<V>(b, w[k], u[k]);
                mul_vec<V>(fw, f[k], w[k]);
                fma_vec<V>(h, f[k], h, b);
                mul_vec<V>(u[k], less, fw);
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) { less[v] = h[v]; b[v] = u[k][v]; }
                fma_vec<V>(h, f[k], h, b);
#pragma unroll
                for (int v = 0; v < V; ++v) u[k][v] = less[v];
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) m.A[v] = f[kSteps - 1][v];
        mul_vec<V>(m.H, f[kSteps - 1], d[kSteps - 1]);
#pragma unroll
        for (int k = kSteps - 2; k >= 0; --k) {
            add_vec<V>(m.H, m.H, d[k]);
            mul_vec<V>(m.H, m.H, f[k]);
            mul_vec<V>(m.A, m.A, f[k]);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) m.A[v] = held<V, GATE>(m.A[v]);
        }
        in.next();
        saved(i0 - span, hs);
        float q[V];
        joiner.join(m, carry, q);
        const long long t0 = p.reverse ? at.len - 1 - i0 : i0;
        if (n == kSteps) {
            const long long last = p.reverse ? t0 - (kSteps - 1) : t0 + kSteps - 1;
            T *qa = pda + last * p.da_t, *qx = pdx + last * p.h_t;
#pragma unroll
            for (int k = kSteps - 1; k >= 0; --k) {
                float oa[V], ox[V], g[V];
                add_vec<V>(g, d[k], q);
                mul_vec<V>(oa, g, u[k]);
                mul_vec<V>(ox, g, w[k]);
                mul_vec<V>(q, g, f[k]);
                store_vec<T, V>(qa, oa);
                store_vec<T, V>(qx, ox);
                qa -= sign * p.da_t;
                qx -= sign * p.h_t;
            }
        } else if (idle) {
            const float zero[V] = {};
            const int rows = Place<V>::count(i0, at.end);
            for (int k = 0; k < rows; ++k) {
                store_vec<T, V>(pda + (i0 + k) * p.da_t, zero);
                store_vec<T, V>(pdx + (i0 + k) * p.h_t, zero);
            }
        } else {
            const int rows = Place<V>::count(i0, at.end);
#pragma unroll
            for (int k = kSteps - 1; k >= 0; --k) {
                float oa[V], ox[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float g = d[k][v] + q[v];
                    oa[v] = k < n ? g * u[k][v] : 0.0f;
                    ox[v] = k < n ? g * w[k][v] : 0.0f;
                    q[v] = f[k][v] * g;
                }
                if (k < rows) {
                    const long long t = k < n ? (p.reverse ? t0 - k : t0 + k) : i0 + k;
                    store_vec<T, V>(pda + t * p.da_t, oa);
                    store_vec<T, V>(pdx + t * p.h_t, ox);
                }
            }
        }
    }
    if (p.hT && at.live && joiner.rank == 0 && threadIdx.x < L::kLanes) store_vec<float, V>(p.hT + at.bd, carry);
    joiner.leave();
}

template <typename T, int V, bool GATE>
cudaError_t launch(LinrecArgs &p, bool backward, int sms, cudaStream_t st)
{
    typedef Lay<V> L;
    const void *fn = backward ? (const void *)linrec_backward_kernel<T, V, GATE> : (const void *)linrec_forward_kernel<T, V, GATE>;
    const long long groups = ((long long)p.B * p.nvec + L::kLanes - 1) / L::kLanes, need = ((long long)p.T + L::kWarpSteps - 1) / L::kWarpSteps;
    // warps of a CTA: no more than there are steps for
    const int warps = need >= kThreads / 32 ? kThreads / 32 : need > 1 ? (int)need : 1;
    // CTAs of a cluster: two for each SM, no more than there are steps for; 16 (which few places on the chip can hold) only
    // where 8 do not reach every SM.  us by CTAs a cluster, bf16: 47 groups of channels (4096 x 1 x 1500) 1: 53.6, 2: 34.6, 4: 24.9, 8: 20.4, 16: 32.4;
    // 94 groups (1024 x 2 x 1500) 1: 15.1, 2: 12.8, 4: 10.0, 8: 13.2; 300 groups (400 x 12 x 800) 1: 11.0, 2: 15.5; 4 groups (65536 x 1 x 120) 8: 150, 16: 93.
    // Gradients, of which fewer CTAs fit an SM, would be faster with half as many: 4096 x 1 x 1500 4: 33.5, 8: 38.3; 400 x 4 x 800 1: 8.5, 4: 12.7.
    int csize = 1;
    while (csize < kMaxCluster && groups * csize < (csize < 8 ? 2ll : 1ll) * sms && (long long)warps * csize < need) csize *= 2;
    p.csize = csize;
    if (groups * csize > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(groups * csize));
    cfg.blockDim = dim3((unsigned)(warps * 32));
    cfg.dynamicSmemBytes = backward ? Ahead<T, V, 3, GATE>::kSmem : Ahead<T, V, 2, GATE>::kSmem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = csize;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = csize > 1 ? 1 : 0;
    static std::atomic<unsigned long long> prepared[2];
    const cudaError_t e = prepare_kernel(fn, prepared[backward], (int)cfg.dynamicSmemBytes, true);
    if (e != cudaSuccess) return e;
    void *args[] = {&p};
    return cudaLaunchKernelExC(&cfg, fn, args);
}

template <typename T, int V>
cudaError_t by_gate(LinrecArgs &p, bool backward, int sms, cudaStream_t st)
{
    p.nvec = p.D / V;
    return p.gate ? launch<T, V, true>(p, backward, sms, st) : launch<T, V, false>(p, backward, sms, st);
}

template <typename T>
cudaError_t by_vector(LinrecArgs &p, bool backward, int sms, cudaStream_t st)
{
    // the widest vector, of up to four channels, that divides them and to which every matrix is aligned
    int v = 4;
    while (p.D % v) v /= 2;
    auto matrix = [&](const void *q, long long t, long long b, int es) {
        while (v > 1 && q && ((uintptr_t)q % (v * es) || t % v || b % v)) v /= 2;
    };
    matrix(p.a, p.a_t, p.a_b, sizeof(T));
    matrix(p.x, p.x_t, p.x_b, sizeof(T));
    matrix(p.h, p.h_t, p.h_b, sizeof(T));
    matrix(p.dh, p.dh_t, p.dh_b, sizeof(T));
    matrix(p.da, p.da_t, p.da_b, sizeof(T));
    matrix(p.hT, 0, 0, 4);
    matrix(p.states, 0, 0, 4);
    int wide_v;
    if (linrec_wide_serves(p, v, sizeof(T) == 2, backward, sms, wide_v)) return launch_linrec_wide(p, wide_v, sizeof(T) == 2, backward, st);
    constexpr int kMost = 8 / sizeof(T);
    if (v >= kMost) return by_gate<T, kMost>(p, backward, sms, st);
    return v == 2 ? by_gate<T, 2>(p, backward, sms, st) : by_gate<T, 1>(p, backward, sms, st);
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

long long linrec_workspace(int chunks, int B, int D) { return chunks > 1 ? (2ll * chunks + 1) * B * D : 0; }

int take_workspace(LinrecArgs &p, float *workspace, long long floats, const Failure &fail)
{
    p.chunks = linrec_chunks(p.T, p.B, p.D, p.chunk_len);
    p.maps = workspace;
    if (p.chunks > 1 && (!workspace || !aligned_to(workspace, 4) || floats < linrec_workspace(p.chunks, p.B, p.D)))
        return fail(LSTM_ERR_INVALID, "bad argument: the workspace is smaller than lstm_linear_recurrence_workspace says");
    return LSTM_OK;
}

bool aligned(const void *p, int dtype) { return aligned_to(p, bytes_of(dtype)); }

}  // namespace
}  // namespace lstm

using namespace lstm;

extern "C" {

long long lstm_linear_recurrence_workspace(int T, int B, int D)
{
    if (T < 0 || B < 0 || D < 1) return -1;
    int chunk_len = 0;
    const int chunks = linrec_chunks(T, B, D, chunk_len);
    return linrec_workspace(chunks, B, D);
}

int lstm_linear_recurrence(const void *a, long long a_t, long long a_b, const void *x, long long x_t, long long x_b, const float *h0,
                           const int *lengths, int T, int B, int D, int dtype, int flags, void *h, long long h_t, long long h_b, float *hT,
                           float *states, float *workspace, long long workspace_floats, void *cuda_stream, char *err, int errlen)
{
    const Failure fail{err, errlen};
    if (const int rc = check(a, x, T, B, D, dtype, flags, fail)) return rc;
    if (T > 0 && B > 0 && !h) return fail(LSTM_ERR_INVALID, "bad argument: h must be given");
    if (!aligned(a, dtype) || !aligned(x, dtype) || !aligned(h, dtype) || !aligned(h0, LSTM_F32) || !aligned(hT, LSTM_F32) ||
        !aligned(states, LSTM_F32) || !aligned(lengths, LSTM_F32))
        return fail(LSTM_ERR_INVALID, "bad argument: a pointer is not aligned to its elements");
    if (!steps_apart(T, B, D, h_t, h_b)) return fail(LSTM_ERR_INVALID, "bad argument: rows of an output overlap");
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
    if (const int rc = take_workspace(p, workspace, workspace_floats, fail)) return rc;
    return run(p, dtype, false, (cudaStream_t)cuda_stream, fail);
}

int lstm_linear_recurrence_backward(const void *a, long long a_t, long long a_b, const void *x, long long x_t, long long x_b,
                                    const float *states, const void *dh, long long dh_t, long long dh_b, const float *dhT,
                                    const int *lengths, int T, int B, int D, int dtype, int flags, void *da, long long da_t, long long da_b,
                                    void *dx, long long dx_t, long long dx_b, float *dh0, float *workspace, long long workspace_floats,
                                    void *cuda_stream, char *err, int errlen)
{
    const Failure fail{err, errlen};
    if (const int rc = check(a, x, T, B, D, dtype, flags, fail)) return rc;
    if (T > 0 && B > 0 && (!states || !dh || !da || !dx)) return fail(LSTM_ERR_INVALID, "bad argument: states, dh, da and dx must be given");
    if (!aligned(a, dtype) || !aligned(x, dtype) || !aligned(dh, dtype) || !aligned(da, dtype) || !aligned(dx, dtype) ||
        !aligned(states, LSTM_F32) || !aligned(dhT, LSTM_F32) || !aligned(dh0, LSTM_F32) || !aligned(lengths, LSTM_F32))
        return fail(LSTM_ERR_INVALID, "bad argument: a pointer is not aligned to its elements");
    if (!steps_apart(T, B, D, da_t, da_b) || !steps_apart(T, B, D, dx_t, dx_b)) return fail(LSTM_ERR_INVALID, "bad argument: rows of an output overlap");
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
    if (const int rc = take_workspace(p, workspace, workspace_floats, fail)) return rc;
    return run(p, dtype, true, (cudaStream_t)cuda_stream, fail);
}

}  // extern "C"
