// The gated linear recurrence for many channels: a CTA has 32 vectors of channels side by side (whole lines of memory) and walks over
// time alone; its warps hold consecutive spans of a few steps.  Spans become maps h -> A h + H (see linrec.cu), every warp leaves
// its own in shared memory, one thread per channel runs through them with the channel's carry and leaves each warp the state in front
// of its span.  Two barriers a round and about 1.5 instructions an element for the joining; few registers, so that enough warps
// are resident to keep the memory busy, which is what bounds it: 2048 x 32 x 1500 of bf16 takes 109 us, 0.82 of the copy rate
// (the kernels of linrec.cu, which can spread one sequence over a cluster, 165).
//
// Few channels and many steps: time is cut into chunks that run side by side like further sequences.  A first kernel reduces every
// chunk to its map (reading the inputs once more than they would have to be, and nothing of what the second one writes), and in front
// of its first round a CTA of the second runs through the maps of the chunks before its own.
//
// Backward: a round's spans begin at saved states, so the same pass over the maps gives the states in front of the spans (from the
// saved ones, forwards) and the gradients that arrive behind them (from the carry, backwards).
#include "../../include/lstm_b200.h"
#include "linrec_parts.cuh"

#include <algorithm>
#include <type_traits>

namespace lstm {
namespace {

// Steps of a warp's span, threads of a CTA, CTAs of an SM, and where inputs wait, for vectors of V channels.
// Four bf16 lie in shared memory two spans ahead (in registers: 2048 x 32 x 1500 151 us instead of 109); two or one wait in registers
// (4096 x 8 x 1502 of fp32 in shared memory: 173 us instead of 113).  Four fp32 are not served: 16384 x 1500 135 us, with two 90.
template <typename T, int V, bool BACK> struct Shape;
template <typename T> struct Shape<T, 4, false> { static constexpr int kSteps = 4, kThreads = 128, kResident = 5, kDepth = 2; };
template <typename T> struct Shape<T, 2, false> { static constexpr int kSteps = 8, kThreads = 256, kResident = 2, kDepth = 0; };
template <typename T> struct Shape<T, 1, false> { static constexpr int kSteps = 16, kThreads = 128, kResident = 4, kDepth = 0; };
template <typename T> struct Shape<T, 4, true> { static constexpr int kSteps = 4, kThreads = 128, kResident = 4, kDepth = 2; };
template <typename T> struct Shape<T, 2, true> { static constexpr int kSteps = 4, kThreads = 256, kResident = 2, kDepth = 0; };
template <typename T> struct Shape<T, 1, true> { static constexpr int kSteps = 8, kThreads = 128, kResident = 4, kDepth = 0; };

template <typename T, int V, int N, bool GATE, bool BACK, typename S = Shape<T, V, BACK>>
using Inputs = std::conditional_t<S::kDepth == 0, InRegisters<T, V, N, GATE, S::kSteps>, InShared<T, V, N, GATE, S::kSteps, S::kThreads, S::kDepth ? S::kDepth : 1>>;

// a lane's channels of one chunk of time, and the one channel whose carry a thread keeps
template <int V>
struct Channels {
    int b, d, len;              // len: steps of the sequence
    int off, stop, end;         // the chunk's first step, its last of the sequence and of the batch (0 where there is no such channel)
    long long bd, BD;
    bool live;
    long long own, own_map;     // channel threadIdx.x of the CTA: index into [B][D] (-1: none) and into [chunks][B][D]
    int own_chunk;
    __device__ explicit Channels(const LinrecArgs &p)
    {
        const long long all = (long long)p.chunks * p.B * p.nvec, vec = (long long)blockIdx.x * 32 + (threadIdx.x & 31);
        live = vec < all;
        const long long cb = live ? vec / p.nvec : 0;
        const int chunk = (int)(cb / p.B);
        b = (int)(cb % p.B);
        d = live ? (int)(vec % p.nvec) * V : 0;
        len = !live ? 0 : p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
        off = chunk * p.chunk_len;
        end = live ? (int)min((long long)p.T, (long long)off + p.chunk_len) : 0;
        stop = min(len, end);
        bd = (long long)b * p.D + d;
        BD = (long long)p.B * p.D;
        const long long mine = (long long)blockIdx.x * 32 + threadIdx.x / V;
        own = own_map = -1;
        own_chunk = 0;
        if (threadIdx.x < 32 * V && mine < all) {
            const long long mcb = mine / p.nvec;
            const int md = (int)(mine % p.nvec) * V + threadIdx.x % V;
            own_chunk = (int)(mcb / p.B);
            own = mcb % p.B * p.D + md;
            own_map = mcb * p.D + md;
        }
    }
};

// The carry of a thread's channel in front of its chunk: the initial one behind the maps of the chunks on the way.  With several chunks the
// first kernel has copied the initial ones behind the maps: the last chunk may write the final state over them while others begin.
__device__ __forceinline__ float carry_before(const LinrecArgs &p, long long own, int chunk, bool backward)
{
    if (own < 0) return 0.0f;
    const long long BD = (long long)p.B * p.D, plane = p.chunks * BD;
    float carry = p.chunks > 1 ? p.maps[2 * plane + own] : p.h0 ? p.h0[own] : 0.0f;
    const int way = backward ? p.chunks - 1 - chunk : chunk;
#pragma unroll 8
    for (int i = 0; i < way; ++i) {
        const float *m = p.maps + (backward ? p.chunks - 1 - i : i) * BD + own;
        carry = fmaf(m[0], carry, m[plane]);
    }
    return carry;
}

// The map of each chunk: of h (forward, from a and x), of what reaches the state in front of it (backward, from a and dh).  A warp has a
// quarter of the chunk and four channels a lane, or as many as a vector has; the four meet once, at the end.
template <typename T, int V, bool GATE, bool BACK>
__global__ void __launch_bounds__(128, 5) linrec_chunk_maps_kernel(const __grid_constant__ LinrecArgs p)
{
    constexpr int kSteps = 4, kC = 32 * V;
    typedef std::conditional_t<sizeof(T) * V == 2, InRegisters<T, V, 2, GATE, kSteps>, InShared<T, V, 2, GATE, kSteps, 128, 2>> In;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ __align__(16) float mapA[4][kC], mapH[4][kC];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Channels<V> at(p);
    const long long sign = p.reverse ? -1 : 1, way = BACK ? -kSteps : kSteps;
    const long long sa = sign * p.a_t, sx = sign * (BACK ? p.dh_t : p.x_t);
    const long long step[2] = {sa, sx};
    const int quarter = p.chunk_len / 4;
    long long ahead = at.off + warp * quarter + (BACK ? quarter - kSteps : 0);
    const long long first = p.reverse ? at.len - 1 - ahead : ahead;
    const T *from[2] = {(const T *)p.a + at.b * p.a_b + at.d + first * p.a_t,
                        BACK ? (const T *)p.dh + at.b * p.dh_b + at.d + first * p.dh_t : (const T *)p.x + at.b * p.x_b + at.d + first * p.x_t};
    In in(smem);
    int left = quarter;                 // steps of the quarter that are still to be fetched
    auto fetch = [&]() {
        in.fetch(from, step, left > 0 ? count_steps<kSteps>(ahead, at.stop) : 0);
        left -= kSteps;
        ahead += way;
        from[0] += way * sa;
        from[1] += way * sx;
    };
#pragma unroll
    for (int i = 0; i < In::kDepth; ++i) fetch();
    float A[V], H[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { A[v] = 1.0f; H[v] = 0.0f; }
    for (int i = 0; i < quarter; i += kSteps) {
        in.next_if_registers();
        fetch();
        in.arrived();
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
            const int k = BACK ? kSteps - 1 - kk : kk;
            const Vec<T, V> ra = in.get_vec(0, k), rx = in.get_vec(1, k);
            float f[V], x[V];
#pragma unroll
            for (int v = 0; v < V; ++v) { f[v] = get<T, V>(ra, v); x[v] = get<T, V>(rx, v); }
            if (GATE) {
                float w[V];
                gate_vec<T, V>(f, f, w);
                if (!BACK) mul_vec<V>(x, x, w);
            }
            if (BACK) {
                add_vec<V>(H, H, x);
                mul_vec<V>(H, H, f);
            } else {
                fma_vec<V>(H, f, H, x);
            }
            mul_vec<V>(A, A, f);
        }
        in.next();
#pragma unroll
        for (int v = 0; v < V; ++v) A[v] = held<V, GATE>(A[v]);
    }
    store_vec<float, V>(&mapA[warp][lane * V], A);
    store_vec<float, V>(&mapH[warp][lane * V], H);
    __syncthreads();
    if (at.own_map >= 0) {
        float a = 1.0f, h = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int w = BACK ? 3 - i : i;
            h = fmaf(mapA[w][threadIdx.x], h, mapH[w][threadIdx.x]);
            a = held<V, GATE>(a * mapA[w][threadIdx.x]);
        }
        if (at.own_chunk == 0) p.maps[2ll * p.chunks * at.BD + at.own] = p.h0 ? p.h0[at.own] : 0.0f;
        p.maps[at.own_map] = a;
        p.maps[(long long)p.chunks * at.BD + at.own_map] = h;
    }
}

template <typename T, int V, bool GATE>
__global__ void __launch_bounds__(Shape<T, V, false>::kThreads, Shape<T, V, false>::kResident) linrec_wide_forward_kernel(const __grid_constant__ LinrecArgs p)
{
    typedef Shape<T, V, false> S;
    constexpr int kSteps = S::kSteps, kWarps = S::kThreads / 32, kSpan = kWarps * kSteps, kC = 32 * V;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ __align__(16) float mapA[kWarps][kC], mapH[kWarps][kC], front[kWarps][kC];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Channels<V> at(p);
    const long long sign = p.reverse ? -1 : 1;
    const long long step[2] = {sign * p.a_t, sign * p.x_t}, jump[2] = {kSpan * step[0], kSpan * step[1]}, out_step = sign * p.h_t, out_jump = kSpan * out_step;
    long long i0 = at.off + warp * kSteps, ahead = i0;
    const long long first = p.reverse ? at.len - 1 - i0 : i0;
    const T *from[2] = {(const T *)p.a + at.b * p.a_b + at.d + first * p.a_t, (const T *)p.x + at.b * p.x_b + at.d + first * p.x_t};
    T *ph = (T *)p.h + at.b * p.h_b + at.d, *out = ph + first * p.h_t;
    typedef Inputs<T, V, 2, GATE, false> In;
    In in(smem);
    auto fetch = [&]() {
        in.fetch(from, step, count_steps<kSteps>(ahead, at.stop));
        ahead += kSpan;
        from[0] += jump[0];
        from[1] += jump[1];
    };
#pragma unroll
    for (int i = 0; i < In::kDepth; ++i) fetch();
    float carry = carry_before(p, at.own, at.own_chunk, false);
    for (long long base = 0; base < p.chunk_len; base += kSpan, i0 += kSpan, out += out_jump) {
        const int n = count_steps<kSteps>(i0, at.stop);
        in.next_if_registers();
        fetch();
        in.arrived();
        float f[kSteps][V], add[kSteps][V];
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const Vec<T, V> ra = in.get_vec(0, k), rx = in.get_vec(1, k);
#pragma unroll
            for (int v = 0; v < V; ++v) { f[k][v] = get<T, V>(ra, v); add[k][v] = get<T, V>(rx, v); }
            if (GATE) {
                float w[V];
                gate_vec<T, V>(f[k], f[k], w);
                mul_vec<V>(add[k], add[k], w);
            }
        }
        in.next();
        float A[V], H[V];
#pragma unroll
        for (int v = 0; v < V; ++v) A[v] = f[0][v];
        first_added<V, GATE>(H, f[0], add[0]);
#pragma unroll
        for (int k = 1; k < kSteps; ++k) {
            fma_vec<V>(H, f[k], H, add[k]);
            mul_vec<V>(A, A, f[k]);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) A[v] = held<V, GATE>(A[v]);
        store_vec<float, V>(&mapA[warp][lane * V], A);
        store_vec<float, V>(&mapH[warp][lane * V], H);
        __syncthreads();
        if (threadIdx.x < kC) {
            float a[kWarps], h[kWarps];
#pragma unroll
            for (int w = 0; w < kWarps; ++w) { a[w] = mapA[w][threadIdx.x]; h[w] = mapH[w][threadIdx.x]; }
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                front[w][threadIdx.x] = carry;
                carry = fmaf(a[w], carry, h[w]);
            }
        }
        __syncthreads();            // from here the maps may be written again; `front` is behind the next round's first barrier, when all have read it
        const Vec<float, V> begin = load_vec<float, V>(&front[warp][lane * V]);
        float h[V];
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = get<float, V>(begin, v);
        if (p.states && i0 < at.end && i0 % LSTM_LINREC_SEGMENT == 0)
            store_vec<float, V>(p.states + i0 / LSTM_LINREC_SEGMENT * at.BD + at.bd, h);
        if (n == kSteps) {
            T *q = out;
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                fma_vec<V>(h, f[k], h, add[k]);
                store_vec<T, V>(q, h);
                q += out_step;
            }
        } else {
            // steps behind a sequence's end lie at their own place in either direction
            const int rows = count_steps<kSteps>(i0, at.end);
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                float o[V];
                fma_vec<V>(h, f[k], h, add[k]);
#pragma unroll
                for (int v = 0; v < V; ++v) o[v] = k < n ? h[v] : 0.0f;
                if (k < rows) store_vec<T, V>(k < n ? out + k * out_step : ph + (i0 + k) * p.h_t, o);
            }
        }
    }
    if (p.hT && at.own >= 0 && at.own_chunk == p.chunks - 1) p.hT[at.own] = carry;
}

template <typename T, int V, bool GATE>
__global__ void __launch_bounds__(Shape<T, V, true>::kThreads, Shape<T, V, true>::kResident) linrec_wide_backward_kernel(const __grid_constant__ LinrecArgs p)
{
    typedef Shape<T, V, true> S;
    constexpr int kSteps = S::kSteps, kWarps = S::kThreads / 32, kSpan = kWarps * kSteps, kC = 32 * V, kStates = kSpan / LSTM_LINREC_SEGMENT;
    static_assert(kSpan % LSTM_LINREC_SEGMENT == 0 && LSTM_LINREC_SEGMENT % kSteps == 0, "a round begins at a saved state");
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ __align__(16) float mapA[kWarps][kC], mapH[kWarps][kC], mapQ[kWarps][kC], front[kWarps][kC], behind[kWarps][kC];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Channels<V> at(p);
    const long long sign = p.reverse ? -1 : 1;
    const long long step[3] = {sign * p.a_t, sign * p.x_t, sign * p.dh_t}, jump[3] = {kSpan * step[0], kSpan * step[1], kSpan * step[2]};
    const long long rounds = ((long long)p.chunk_len + kSpan - 1) / kSpan;
    long long base = (rounds - 1) * kSpan, i0 = at.off + base + warp * kSteps, ahead = i0;
    const long long first = p.reverse ? at.len - 1 - i0 : i0;
    const T *from[3] = {(const T *)p.a + at.b * p.a_b + at.d + first * p.a_t, (const T *)p.x + at.b * p.x_b + at.d + first * p.x_t,
                        (const T *)p.dh + at.b * p.dh_b + at.d + first * p.dh_t};
    T *pda = (T *)p.da + at.b * p.da_b + at.d, *pdx = (T *)p.h + at.b * p.h_b + at.d;
    typedef Inputs<T, V, 3, GATE, true> In;
    In in(smem);
    auto fetch = [&]() {
        in.fetch(from, step, count_steps<kSteps>(ahead, at.stop));
        ahead -= kSpan;
#pragma unroll
        for (int i = 0; i < 3; ++i) from[i] -= jump[i];
    };
#pragma unroll
    for (int i = 0; i < In::kDepth; ++i) fetch();
    float saved[kStates];
    auto fetch_states = [&](long long of) {
#pragma unroll
        for (int s = 0; s < kStates; ++s) {
            const long long i = (long long)at.own_chunk * p.chunk_len + of + s * LSTM_LINREC_SEGMENT;
            saved[s] = at.own >= 0 && i >= 0 && i < p.T ? p.states[i / LSTM_LINREC_SEGMENT * at.BD + at.own] : 0.0f;
        }
    };
    fetch_states(base);
    float carry = carry_before(p, at.own, at.own_chunk, true);      // what reaches the state behind the steps that are left
    for (; base >= 0; base -= kSpan, i0 -= kSpan) {
        const int n = count_steps<kSteps>(i0, at.stop);
        in.next_if_registers();
        fetch();
        in.arrived();
        float f[kSteps][V], w[kSteps][V];
        float A[V], H[V], Q[V];
#pragma unroll
        for (int v = 0; v < V; ++v) { A[v] = 1.0f; H[v] = Q[v] = 0.0f; }
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const Vec<T, V> ra = in.get_vec(0, k), rx = in.get_vec(1, k);
            float x[V];
#pragma unroll
            for (int v = 0; v < V; ++v) { f[k][v] = get<T, V>(ra, v); x[v] = get<T, V>(rx, v); w[k][v] = 1.0f; }
            if (GATE) {
                gate_vec<T, V>(f[k], f[k], w[k]);
                mul_vec<V>(x, x, w[k]);
            }
            fma_vec<V>(H, f[k], H, x);
            mul_vec<V>(A, A, f[k]);
        }
#pragma unroll
        for (int k = kSteps - 1; k >= 0; --k) {
            const Vec<T, V> rd = in.get_vec(2, k);
            float d[V];
#pragma unroll
            for (int v = 0; v < V; ++v) d[v] = get<T, V>(rd, v);
            add_vec<V>(Q, Q, d);
            mul_vec<V>(Q, Q, f[k]);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) A[v] = held<V, GATE>(A[v]);
        store_vec<float, V>(&mapA[warp][lane * V], A);
        store_vec<float, V>(&mapH[warp][lane * V], H);
        store_vec<float, V>(&mapQ[warp][lane * V], Q);
        __syncthreads();
        if (threadIdx.x < kC) {
            float a[kWarps], h[kWarps], q[kWarps], state = 0.0f;
#pragma unroll
            for (int i = 0; i < kWarps; ++i) { a[i] = mapA[i][threadIdx.x]; h[i] = mapH[i][threadIdx.x]; q[i] = mapQ[i][threadIdx.x]; }
#pragma unroll
            for (int i = 0; i < kWarps; ++i) {
                if (i * kSteps % LSTM_LINREC_SEGMENT == 0) state = saved[i * kSteps / LSTM_LINREC_SEGMENT];
                front[i][threadIdx.x] = state;
                state = fmaf(a[i], state, h[i]);
            }
#pragma unroll
            for (int i = kWarps - 1; i >= 0; --i) {
                behind[i][threadIdx.x] = carry;
                carry = fmaf(a[i], carry, q[i]);
            }
            fetch_states(base - kSpan);
        }
        __syncthreads();
        const Vec<float, V> begin = load_vec<float, V>(&front[warp][lane * V]), end = load_vec<float, V>(&behind[warp][lane * V]);
        float h[V], q[V], u[kSteps][V];
#pragma unroll
        for (int v = 0; v < V; ++v) { h[v] = get<float, V>(begin, v); q[v] = get<float, V>(end, v); }
        // da_t = g_t u_t and dx_t = g_t w_t with u = (h_{t-1} - x) f (1 - f), w = 1 - f  (decay: u = h_{t-1}, w = 1)
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const Vec<T, V> rx = in.get_vec(1, k);
            float x[V];
#pragma unroll
            for (int v = 0; v < V; ++v) { x[v] = get<T, V>(rx, v); u[k][v] = GATE ? h[v] - x[v] : h[v]; }
            if (GATE) {
                float fw[V];
                mul_vec<V>(fw, f[k], w[k]);
                mul_vec<V>(u[k], u[k], fw);
                mul_vec<V>(x, x, w[k]);
            }
            fma_vec<V>(h, f[k], h, x);
        }
        const int rows = count_steps<kSteps>(i0, at.end);
        const long long t0 = p.reverse ? at.len - 1 - i0 : i0;
        T *qa = pda + t0 * p.da_t, *qx = pdx + t0 * p.h_t;
#pragma unroll
        for (int k = kSteps - 1; k >= 0; --k) {
            const Vec<T, V> rd = in.get_vec(2, k);
            float oa[V], ox[V], g[V];
#pragma unroll
            for (int v = 0; v < V; ++v) g[v] = get<T, V>(rd, v);
            add_vec<V>(g, g, q);
            mul_vec<V>(oa, g, u[k]);
            mul_vec<V>(ox, g, w[k]);
            mul_vec<V>(q, g, f[k]);
            if (n == kSteps || k < n) {
                store_vec<T, V>(qa + k * sign * p.da_t, oa);
                store_vec<T, V>(qx + k * sign * p.h_t, ox);
            } else if (k < rows) {
                store_raw<T, V>(pda + (i0 + k) * p.da_t, zero_vec<T, V>());
                store_raw<T, V>(pdx + (i0 + k) * p.h_t, zero_vec<T, V>());
            }
        }
        in.next();
    }
    if (p.hT && at.own >= 0 && at.own_chunk == 0) p.hT[at.own] = carry;
}

// Up to four steps (generation): a thread runs through its vector's steps alone, nothing is joined (16 x 1500: 4.5 us -> 1.6).
constexpr int kShort = 4;
template <typename T, int V, bool GATE>
__global__ void __launch_bounds__(64) linrec_short_kernel(const __grid_constant__ LinrecArgs p)
{
    const long long vec = (long long)blockIdx.x * 64 + threadIdx.x;
    if (vec >= (long long)p.B * p.nvec) return;
    const int b = (int)(vec / p.nvec), d = (int)(vec % p.nvec) * V;
    const int len = p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
    const long long bd = (long long)b * p.D + d, sign = p.reverse ? -1 : 1, first = p.reverse ? len - 1 : 0;
    const T *pa = (const T *)p.a + b * p.a_b + d + first * p.a_t, *px = (const T *)p.x + b * p.x_b + d + first * p.x_t;
    T *ph = (T *)p.h + b * p.h_b + d;
    Vec<T, V> ra[kShort], rx[kShort];
    float h[V];
#pragma unroll
    for (int k = 0; k < kShort; ++k) {
        if (k >= p.T) break;
        ra[k] = k < len ? load_vec<T, V>(pa + k * sign * p.a_t) : keep<T, V, GATE>();
        rx[k] = k < len ? load_vec<T, V>(px + k * sign * p.x_t) : zero_vec<T, V>();
    }
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = p.h0 ? p.h0[bd + v] : 0.0f;
    if (p.states && p.T > 0) store_vec<float, V>(p.states + bd, h);      // (no steps: there are no saved states)
#pragma unroll
    for (int k = 0; k < kShort; ++k) {
        if (k >= p.T) break;
        float f[V], x[V];
#pragma unroll
        for (int v = 0; v < V; ++v) { f[v] = get<T, V>(ra[k], v); x[v] = get<T, V>(rx[k], v); }
        if (GATE) {
            float w[V];
            gate_vec<T, V>(f, f, w);
            mul_vec<V>(x, x, w);
        }
        fma_vec<V>(h, f, h, x);
        if (k < len) store_vec<T, V>(ph + (first + k * sign) * p.h_t, h);
        else store_raw<T, V>(ph + k * p.h_t, zero_vec<T, V>());
    }
    if (p.hT) store_vec<float, V>(p.hT + bd, h);
}

template <typename T, int V, bool GATE>
cudaError_t launch(LinrecArgs &p, bool backward, cudaStream_t st)
{
    p.nvec = p.D / V;
    if (!backward && p.T <= kShort) {
        linrec_short_kernel<T, V, GATE><<<(unsigned)(((long long)p.B * p.nvec + 63) / 64), 64, 0, st>>>(p);
        return cudaGetLastError();
    }
    const void *fn = backward ? (const void *)linrec_wide_backward_kernel<T, V, GATE> : (const void *)linrec_wide_forward_kernel<T, V, GATE>;
    const int smem = backward ? Inputs<T, V, 3, GATE, true>::kSmem : Inputs<T, V, 2, GATE, false>::kSmem;
    static std::atomic<unsigned long long> prepared[2];
    const cudaError_t e = prepare_kernel(fn, prepared[backward], smem, false);
    if (e != cudaSuccess) return e;
    const long long groups = ((long long)p.chunks * p.B * p.nvec + 31) / 32;
    if (groups > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    void *args[] = {&p};
    if (p.chunks > 1) {
        const void *maps = backward ? (const void *)linrec_chunk_maps_kernel<T, V, GATE, true> : (const void *)linrec_chunk_maps_kernel<T, V, GATE, false>;
        constexpr int kMapSmem = sizeof(T) * V == 2 ? 0 : InShared<T, V, 2, GATE, 4, 128, 2>::kSmem;
        static std::atomic<unsigned long long> maps_prepared[2];
        cudaError_t e2 = prepare_kernel(maps, maps_prepared[backward], kMapSmem, false);
        if (e2 == cudaSuccess) e2 = cudaLaunchKernel(maps, dim3((unsigned)groups), dim3(128), args, kMapSmem, st);
        if (e2 != cudaSuccess) return e2;
    }
    return cudaLaunchKernel(fn, dim3((unsigned)groups), dim3(backward ? Shape<T, V, true>::kThreads : Shape<T, V, false>::kThreads), args, smem, st);
}
template <typename T>
cudaError_t by_vector(LinrecArgs &p, int v, bool backward, cudaStream_t st)
{
    if constexpr (sizeof(T) == 2)
        if (v == 4) return p.gate ? launch<T, 4, true>(p, backward, st) : launch<T, 4, false>(p, backward, st);
    if (v == 2) return p.gate ? launch<T, 2, true>(p, backward, st) : launch<T, 2, false>(p, backward, st);
    return p.gate ? launch<T, 1, true>(p, backward, st) : launch<T, 1, false>(p, backward, st);
}

}  // namespace

// From here on vectors of two channels, or of one, make some 1.2 CTAs an SM (of 148) by themselves: many channels, without chunks.
static long long many_channels(int v) { return v == 1 ? 5600 : 11000; }

// Chunks pay where channels alone do not fill the chip and the work is large enough for a second launch and a second reading, most of
// which comes from L2 up to some ten million elements.  us, cluster of CTAs (linrec.cu) / chunks: 65536 x 1 x 1500 of bf16 261 / 200,
// backward 529 / 320; 16384 x 1 x 1500 69 / 59; 4096 x 4 x 1000 52 / 41; 65536 x 1 x 256 102 / 48; 4096 x 1 x 1500 20 / 21.
// As many chunks as make some 75000 channels side by side, just under what is resident at once in vectors of four bf16 (65536 x 1500: 36000 228 us, 48000
// 200, 93000 194, 120000 217; backward 342, 320, 336, 340, and 72000 295); fp32 in vectors of two makes several waves of them.  No more than 64: each
// has to run through the maps of those before it.
int linrec_chunks(int T, int B, int D, int &chunk_len)
{
    chunk_len = T;
    const long long channels = (long long)B * D;
    if (channels > many_channels(D % 2 ? 1 : 2) || channels * T < 8000000 || T < 512) return 1;
    const int want = (int)std::min(std::max(75000 / channels, 2ll), 64ll);
    const long long len = (((long long)T + want - 1) / want + 63) / 64 * 64;
    chunk_len = (int)len;
    return (int)((T + len - 1) / len);
}

// Without chunks: vectors of four where they make two CTAs an SM, else of two (or one), from many_channels on.  us, linrec.cu / here: 2048 x 32 x 1500
// of bf16 165 / 110, 400 x 64 x 800 47 / 25, 35 x 20 x 1500 8.7 / 4.9, 512 x 64 x 1501 131 / 77, 4096 x 8 x 1500 of fp32 132 / 113 (188 CTAs of vectors of
// two; with vectors of four, 94 CTAs, 148).  Just above the line 16384 x 4 x 2800 338 / 306, of fp32 476 / 404, backward 682 / 641 and 1004 / 769; 400 x 14 x 800
// 11.2 / 11.1, of fp32 backward 28 / 21; 400 x 7 x 801 13.8 / 12.1.  Bf16 gradients in vectors of one are the exception, 1000 x 7 x 809 46 / 50.  Below it
// 400 x 12 x 800 11.1 / 11.1, of fp32 11.9 / 12.5, 200 x 8 x 700 6.5 / 6.3, and long sequences in chunks.
bool linrec_wide_serves(const LinrecArgs &p, int v, bool bf16, bool backward, int sms, int &wide_v)
{
    const long long channels = (long long)p.chunks * p.B * p.D;
    wide_v = bf16 ? v : std::min(v, 2);
    if (p.T <= kShort && !backward) return true;
    if (wide_v == 4 && (channels / 4 + 31) / 32 < 2 * sms) wide_v = 2;
    return p.chunks > 1 || channels > (bf16 && backward && wide_v == 1 ? 5664 : many_channels(wide_v));
}

cudaError_t launch_linrec_wide(LinrecArgs &p, int v, bool bf16, bool backward, cudaStream_t st)
{
    return bf16 ? by_vector<__nv_bfloat16>(p, v, backward, st) : by_vector<float>(p, v, backward, st);
}

}  // namespace lstm
