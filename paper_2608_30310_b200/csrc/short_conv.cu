// Depthwise causal convolution over K rows, for packed prompts and for single tokens.
//
//     out[t,c] = act(bias[c] + sum_j w[c,j] x[t - K + 1 + j, c])
//
// A thread has VEC neighbouring channels and walks R rows of the packed batch with the last K - 1 rows in registers, so that every
// row is read once, but for the K - 1 rows before a thread's first.  Where a request begins inside the walk, the window is refilled
// from the request's start state, and the same thread writes the request's final state: it has read the start state by then, so that
// both may be the same memory.  Bound by HBM: 2 K + 4 flops and two special-function results a value against 4 bytes moved (bf16).
#include "layers.cuh"

namespace gdn {
namespace {

constexpr int kAhead = 8;              // rows loaded side by side

template <typename T, int K, int VEC>
struct Window {
    float w[K][VEC], bias[VEC], hist[K - 1][VEC];
    bool silu;

    __device__ __forceinline__ void load_weights(const ConvArgs& a, int c)
    {
        silu = a.silu;
        Pack<T, VEC * K> p;
        const T* weight = static_cast<const T*>(a.weight) + (size_t)c * K;
        if (VEC > 1) p = *reinterpret_cast<const Pack<T, VEC * K>*>(weight);
        else
#pragma unroll
            for (int j = 0; j < K; ++j) p.v[j] = weight[j];
#pragma unroll
        for (int v = 0; v < VEC; ++v)
#pragma unroll
            for (int j = 0; j < K; ++j) w[j][v] = widen<T>(p.v[v * K + j]);
        if (a.bias) {
            const Pack<T, VEC> q = *reinterpret_cast<const Pack<T, VEC>*>(static_cast<const T*>(a.bias) + c);
#pragma unroll
            for (int v = 0; v < VEC; ++v) bias[v] = widen<T>(q.v[v]);
        } else {
#pragma unroll
            for (int v = 0; v < VEC; ++v) bias[v] = 0.f;
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int j = 0; j < K - 1; ++j)
#pragma unroll
            for (int v = 0; v < VEC; ++v) hist[j][v] = 0.f;
    }
    __device__ __forceinline__ void set(int j, const Pack<T, VEC>& p)
    {
#pragma unroll
        for (int v = 0; v < VEC; ++v) hist[j][v] = widen<T>(p.v[v]);
    }
    // the next row in, its result out
    __device__ __forceinline__ Pack<T, VEC> step(const Pack<T, VEC>& p)
    {
        Pack<T, VEC> out;
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            const float x = widen<T>(p.v[v]);
            float acc = bias[v];
#pragma unroll
            for (int j = 0; j < K - 1; ++j) acc = fmaf(w[j][v], hist[j][v], acc);
            acc = fmaf(w[K - 1][v], x, acc);
#pragma unroll
            for (int j = 0; j < K - 2; ++j) hist[j][v] = hist[j + 1][v];
            hist[K - 2][v] = x;
            out.v[v] = round_to<T>(silu ? silu_of(acc) : acc);
        }
        return out;
    }
};

template <typename T, int K, int VEC>
__global__ void __launch_bounds__(128) short_conv_kernel(const ConvArgs a, const int rows, const uint32_t vectors, const uint32_t tiles)
{
    using P = Pack<T, VEC>;
    const uint32_t id = blockIdx.x * 128u + threadIdx.x, tile = id / vectors, c = (id - tile * vectors) * VEC;
    allow_successor();
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
    auto walk = [&](int t, int end) {
        for (; t < end; t += kAhead) {
            P p[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (t + i < end) p[i] = row(t + i);
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (t + i < end) *reinterpret_cast<P*>(out + (int64_t)(t + i) * a.out_stride) = win.step(p[i]);
        }
    };

    int n = 0;                                               // the first request that begins at t0 or after it
    for (int hi = N; n < hi;) {
        const int mid = (n + hi) / 2;
        if (a.cu[mid] < t0) n = mid + 1; else hi = mid;
    }
    if (n > 0 && t0 < min(a.cu[n], t1)) {                    // (cu[n] > t0: otherwise it begins here)
        const int begin = a.cu[n - 1], slot = init && t0 - begin < K - 1 ? slot_of(a.init_slots, n - 1, a.num_init, a.status_word) : -1;
        win.clear();
#pragma unroll
        for (int j = 0; j < K - 1; ++j) {
            const int t = t0 - (K - 1) + j;
            if (t >= begin) win.set(j, row(t));
            else if (slot >= 0) win.set(j, *reinterpret_cast<const P*>(init + ((int64_t)slot * (K - 1) + (K - 1 + t - begin)) * a.channels));
        }
        walk(t0, min(a.cu[n], t1));
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
        walk(begin, min(end, t1));
    }
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
    // Rows per thread: the longest walk that still leaves every SM 512 threads.
    int rows = 64;
    while (rows > kAhead && (uint64_t)((a.total_tokens + rows - 1) / rows) * vectors < 148 * 512) rows /= 2;
    const uint64_t tiles = a.total_tokens > 0 ? (uint64_t)(a.total_tokens + rows - 1) / rows : 1, threads = tiles * vectors;
    if (threads > 0xffffffffull - 128) return cudaErrorNotSupported;
    return launch_kernel(short_conv_kernel<T, K, VEC>, (unsigned)((threads + 127) / 128), 128, 0, stream, 1, a, rows, vectors, (uint32_t)tiles);
}

template <typename T>
cudaError_t launch_width(const ConvArgs& a, int width, bool step, cudaStream_t stream)
{
    constexpr int VEC = 4;
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
