// Depthwise causal convolution over K rows, for packed prompts and for single tokens.
//
//     out[t,c] = act(bias[c] + sum_j w[c,j] x[t - K + 1 + j, c])
//
// A thread has VEC neighbouring channels and walks R rows of the packed batch with the last K - 1 rows in registers, so that every
// row is read once, but for the K - 1 rows before a thread's first.  Where a request begins inside the walk, the window is refilled
// from the request's start state, and the same thread writes the request's final state; it also goes on for the K - 1 rows that need the
// start state, past the end of its share if need be.  So no other thread reads the start state, and both may be the same memory.  Bound by HBM, closely followed by the special-function unit (two
// results a value, 61 % busy) and the loads' latency.  Four hits (10,094 rows of 8,192 bf16 channels): 67 us, 4.9 TB/s (62 us in a graph); 51 us at
// the copy rate.  One channel a thread, where the alignment or the number of channels asks for it: 182 us.
#include "layers.cuh"

namespace gdn {
namespace {

constexpr int kRows = 4, kGroups = 4, kResident = 6;   // kResident: CTAs on an SM

// VEC channels as pairs; a single channel is the first half of one
template <int VEC> struct Values {
    static constexpr int N = (VEC + 1) / 2;
    F2 v[N];
};
template <typename T, int VEC> __device__ __forceinline__ Values<VEC> widened(const Pack<T, VEC>& p)
{
    Values<VEC> r;
#pragma unroll
    for (int i = 0; i < Values<VEC>::N; ++i) r.v[i] = pair(widen<T>(p.v[2 * i]), 2 * i + 1 < VEC ? widen<T>(p.v[2 * i + 1 < VEC ? 2 * i + 1 : 0]) : 0.f);
    return r;
}

template <typename T, int K, int VEC>
struct Window {
    static constexpr int N = Values<VEC>::N;
    Values<VEC> w[K], bias, hist[K - 1];
    bool silu;

    __device__ __forceinline__ void load_weights(const ConvArgs& a, int c)
    {
        silu = a.silu;
        const T* weight = static_cast<const T*>(a.weight) + (size_t)c * K;
        T p[VEC * K];                                        // (of channel 0, then of channel 1, ...)
#pragma unroll
        for (int j = 0; j < K; ++j) {                        // in packs as wide as the rows': the alignment that the choice of VEC asks of the weights
            const Pack<T, VEC> q = *reinterpret_cast<const Pack<T, VEC>*>(weight + j * VEC);
#pragma unroll
            for (int v = 0; v < VEC; ++v) p[j * VEC + v] = q.v[v];
        }
#pragma unroll
        for (int j = 0; j < K; ++j) {
            Pack<T, VEC> q;
#pragma unroll
            for (int v = 0; v < VEC; ++v) q.v[v] = p[v * K + j];
            w[j] = widened<T, VEC>(q);
        }
        if (a.bias) bias = widened<T, VEC>(*reinterpret_cast<const Pack<T, VEC>*>(static_cast<const T*>(a.bias) + c));
        else bias = {};
    }
    __device__ __forceinline__ void set(int j, const Pack<T, VEC>& p) { hist[j] = widened<T, VEC>(p); }
    // the next row in, its result out
    __device__ __forceinline__ Pack<T, VEC> step(const Pack<T, VEC>& p)
    {
        const Values<VEC> x = widened<T, VEC>(p);
        Pack<T, VEC> out;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            F2 acc = bias.v[i];
#pragma unroll
            for (int j = 0; j < K - 1; ++j) acc = fma(w[j].v[i], hist[j].v[i], acc);
            acc = fma(w[K - 1].v[i], x.v[i], acc);
            if (silu) acc = silu_of(acc);
            const float2 r = parts(acc);
            out.v[2 * i] = round_to<T>(r.x);
            if (2 * i + 1 < VEC) out.v[2 * i + 1 < VEC ? 2 * i + 1 : 0] = round_to<T>(r.y);
        }
#pragma unroll
        for (int j = 0; j < K - 2; ++j) hist[j] = hist[j + 1];
        hist[K - 2] = x;
        return out;
    }
};

template <typename T, int K, int VEC>
__global__ void __launch_bounds__(128, kResident) short_conv_kernel(const ConvArgs a, const int rows, const uint32_t vectors, const uint32_t tiles)
{
    using P = Pack<T, VEC>;
    const uint32_t id = blockIdx.x * 128u + threadIdx.x, tile = id / vectors, c = (id - tile * vectors) * VEC;
    wait_for_predecessor();
    if (tile >= tiles) return;
    const int N = a.num_seqs, last = (int)min((int64_t)a.cu[N], a.total_tokens);
    const uint32_t end_tile = min((uint32_t)last / rows, tiles - 1);               // the rest is a padded batch's
    if (tile > end_tile) return;
    const int t0 = tile * rows, t1 = tile == end_tile ? last : t0 + rows;
    Window<T, K, VEC> win;
    win.load_weights(a, c);
    const T* x = static_cast<const T*>(a.x) + c;
    T* out = static_cast<T*>(a.out) + c;
    const T* init = a.init_state ? static_cast<const T*>(a.init_state) + c : nullptr;
    T* keep = a.out_state ? static_cast<T*>(a.out_state) + c : nullptr;
    auto row = [&](int t) { return *reinterpret_cast<const P*>(x + (int64_t)t * a.x_stride); };
    // Groups of kRows rows are copied to shared memory kGroups - 1 ahead of the walk: registers for as many loads in flight would leave
    // too few warps.  A thread reads what it copied itself; nothing waits for another.
    __shared__ P ring[kGroups * kRows][128];
    auto walk = [&](int t, int end) {
        const T* from = x + (int64_t)t * a.x_stride;
        T* to = out + (int64_t)t * a.out_stride;
        const int rows_left = end - t, groups = (rows_left + kRows - 1) / kRows;
        auto issue = [&](int g) {
#pragma unroll
            for (int i = 0; i < kRows; ++i, from += a.x_stride)
                if (g * kRows + i < rows_left) {
                    P* dst = &ring[g % kGroups * kRows + i][threadIdx.x];
                    if constexpr (sizeof(P) >= 4) copy_async<sizeof(P)>(dst, from);
                    else *dst = *reinterpret_cast<const P*>(from);
                }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        for (int g = 0; g < kGroups - 1; ++g) issue(g);
        for (int g = 0; g < groups; ++g) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kGroups - 2) : "memory");
            P p[kRows];
#pragma unroll
            for (int i = 0; i < kRows; ++i) p[i] = ring[g % kGroups * kRows + i][threadIdx.x];
            issue(g + kGroups - 1);
            const int here = rows_left - g * kRows;
            if (here >= kRows) {
#pragma unroll
                for (int i = 0; i < kRows; ++i, to += a.out_stride) *reinterpret_cast<P*>(to) = win.step(p[i]);
            } else {
#pragma unroll
                for (int i = 0; i < kRows - 1; ++i, to += a.out_stride)
                    if (i < here) *reinterpret_cast<P*>(to) = win.step(p[i]);
            }
        }
    };

    int n = 0;                                               // the first request that begins at t0 or after it
    for (int hi = N; n < hi;) {
        const int mid = (n + hi) / 2;
        if (a.cu[mid] < t0) n = mid + 1; else hi = mid;
    }
    if (n > 0) {                                             // a request that began before: its first K - 1 rows are not this walk's
        const int begin = a.cu[n - 1], from = max(t0, begin + K - 1), end = min(a.cu[n], t1);
        if (from < end) {
#pragma unroll
            for (int j = 0; j < K - 1; ++j) win.set(j, row(from - (K - 1) + j));
            walk(from, end);
        }
    }
    for (; n < N; ++n) {
        const int begin = a.cu[n], end = min(a.cu[n + 1], last);
        if (begin >= t1 && tile != end_tile) break;
        const int from = init ? slot_of(a.init_slots, n, a.num_init, a.status_word) : -1;
        const int to = keep ? slot_of(a.out_slots, n, a.num_out, a.status_word) : -1;
        P h[K - 1];
#pragma unroll
        for (int j = 0; j < K - 1; ++j) {
            if (from >= 0) h[j] = *reinterpret_cast<const P*>(init + ((int64_t)from * (K - 1) + j) * a.channels);
            else
#pragma unroll
                for (int v = 0; v < VEC; ++v) h[j].v[v] = round_to<T>(0.f);
            win.set(j, h[j]);
        }
        if (to >= 0) {
            T* s = keep + (int64_t)to * (K - 1) * a.channels;
#pragma unroll
            for (int j = 0; j < K - 1; ++j) {                // row j of the last K - 1 of (start state, rows)
                const int t = end - (K - 1) + j;
                P p;
                if (t >= begin) p = row(t);
                else {
#pragma unroll
                    for (int i = 0; i < K - 1; ++i)
                        if (i == end - begin + j) p = h[i];
                }
                *reinterpret_cast<P*>(s + (int64_t)j * a.channels) = p;
            }
        }
        walk(begin, min(end, max(t1, begin + K - 1)));       // (as many rows as need the start state)
    }
    allow_successor();                                       // (at the end: an early successor would be spread over the SMs that are free by then)
}

// One token per request: the window is the request's state.
template <typename T, int K, int VEC>
__global__ void __launch_bounds__(128) short_conv_step_kernel(const ConvArgs a, const uint32_t vectors)
{
    using P = Pack<T, VEC>;
    const uint32_t id = blockIdx.x * 128u + threadIdx.x, n = id / vectors, c = (id - n * vectors) * VEC;
    allow_successor();
    wait_for_predecessor();
    if (n >= (uint32_t)a.num_seqs) return;
    const int slot = slot_of(a.init_slots, n, min(a.num_init, a.num_out), a.status_word);
    if (slot < 0) return;
    const int64_t at = (int64_t)slot * (K - 1) * a.channels + c;
    const T* in = static_cast<const T*>(a.init_state) + at;
    T* keep = static_cast<T*>(a.out_state) + at;
    P h[K - 1];
#pragma unroll
    for (int j = 0; j < K - 1; ++j) h[j] = *reinterpret_cast<const P*>(in + (int64_t)j * a.channels);
    const P x = *reinterpret_cast<const P*>(static_cast<const T*>(a.x) + (int64_t)n * a.x_stride + c);
    Window<T, K, VEC> win;
    win.load_weights(a, c);
#pragma unroll
    for (int j = 0; j < K - 1; ++j) win.set(j, h[j]);
#pragma unroll
    for (int j = 0; j < K - 1; ++j) *reinterpret_cast<P*>(keep + (int64_t)j * a.channels) = j + 1 < K - 1 ? h[j + 1 < K - 1 ? j + 1 : 0] : x;
    *reinterpret_cast<P*>(static_cast<T*>(a.out) + (int64_t)n * a.out_stride + c) = win.step(x);
}

template <typename T, int K, int VEC>
cudaError_t launch(const ConvArgs& a, bool step, cudaStream_t stream)
{
    const uint32_t vectors = a.channels / VEC;
    if (step) {
        const uint64_t threads = (uint64_t)a.num_seqs * vectors;
        if (threads > 0xffffffffull - 128) return cudaErrorNotSupported;
        return launch_kernel(short_conv_step_kernel<T, K, VEC>, (unsigned)((threads + 127) / 128), 128, 0, stream, 1, a, vectors);
    }
    // Rows per thread: two rounds of resident CTAs, but at least eight rows (us with one / two / four rounds: four hits of 8,192 channels 62.8 / 62.0 /
    // 62.0, the same in three calls of fewer channels 75 / 77 / 81, 32 hits 472 / 440 / 430; 410 rows 7.3 / 7.4 / 7.1).
    const int64_t threads_wanted = 2 * 148ll * kResident * 128;
    int rows = (int)((a.total_tokens * (int64_t)vectors + threads_wanted - 1) / threads_wanted);
    rows = rows < 8 ? 8 : (rows + kRows - 1) / kRows * kRows;
    const uint64_t tiles = a.total_tokens > 0 ? (uint64_t)(a.total_tokens + rows - 1) / rows : 1, threads = tiles * vectors;
    if (threads > 0xffffffffull - 128) return cudaErrorNotSupported;
    return launch_kernel(short_conv_kernel<T, K, VEC>, (unsigned)((threads + 127) / 128), 128, 0, stream, 1, a, rows, vectors, (uint32_t)tiles);
}

template <typename T>
cudaError_t launch_width(const ConvArgs& a, int width, bool step, cudaStream_t stream)
{
    constexpr int VEC = 4;
    static_assert(alignof(Pack<T, VEC>) == VEC * sizeof(T), "what the kernels load at once is what is checked here");
    const uintptr_t all = (uintptr_t)a.x | (uintptr_t)a.weight | (uintptr_t)a.bias | (uintptr_t)a.init_state | (uintptr_t)a.out |
                          (uintptr_t)a.out_state | (uintptr_t)((a.x_stride | a.out_stride) * (int64_t)sizeof(T));
    const bool vec = (all & (VEC * sizeof(T) - 1)) == 0 && a.channels % VEC == 0;
    switch (width) {
        case 2: return vec ? launch<T, 2, VEC>(a, step, stream) : launch<T, 2, 1>(a, step, stream);
        case 3: return vec ? launch<T, 3, VEC>(a, step, stream) : launch<T, 3, 1>(a, step, stream);
        case 4: return vec ? launch<T, 4, VEC>(a, step, stream) : launch<T, 4, 1>(a, step, stream);
    }
    return cudaErrorNotSupported;
}

}  // namespace

cudaError_t launch_conv(const ConvArgs& a, int io_dtype, int width, bool step, cudaStream_t stream)
{
    return io_dtype == GDN_BF16 ? launch_width<__nv_bfloat16>(a, width, step, stream) : launch_width<float>(a, width, step, stream);
}

}  // namespace gdn
