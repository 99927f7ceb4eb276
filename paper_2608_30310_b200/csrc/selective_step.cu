// One token of the selective scan per request, from and to a state in memory.
//
// Bound by HBM: every state is read and written once (8 bytes), for one exponential and five flops.  A thread has eight states of a
// channel (32 bytes, one sector, each way) and serves R requests side by side with its decays in registers; S / 8 lanes share a channel.
#include "selective_scan.cuh"

namespace gdn {
namespace scan {
namespace {

template <typename T> __device__ __forceinline__ void load8(const T* p, bool packed, float (&v)[8])
{
    if (packed) load_values<T, 8>(p, v);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = widen<T>(p[i]);
}

// packed: rows of b and c begin on 16 bytes
template <typename T, int S, int R>
__global__ void __launch_bounds__(128) selective_step_kernel(const ScanArgs a, const uint32_t per_request, const bool packed)
{
    constexpr int LN = S / 8;
    const uint32_t id = blockIdx.x * 128u + threadIdx.x, set = id / per_request, at = id - set * per_request;
    const int ch = at / LN, ln = at % LN;                    // (per_request is a multiple of 32: a channel's lanes share a warp)
    allow_successor();
    wait_for_predecessor();
    if ((int64_t)set * R >= a.num_seqs) return;
    const bool real = ch < a.channels;
    int slot[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int n = set * R + i;
        slot[i] = real && n < a.num_seqs ? slot_of(a.init_slots, n, min(a.num_init, a.num_out), a.status_word) : -1;
    }
    float h[R][8], a2[8];
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (slot[i] >= 0) load_values<float, 8>(a.init_state + ((int64_t)slot[i] * a.channels + ch) * S + ln * 8, h[i]);
    float bias = 0.f, skip = 0.f;
    if (real) {
        load_values<float, 8>(a.a + (int64_t)ch * S + ln * 8, a2);
        if (a.dt_bias) bias = a.dt_bias[ch];
        if (a.d) skip = a.d[ch];
    }
#pragma unroll
    for (int s = 0; s < 8; ++s) a2[s] *= kLog2e;
    const int group = real ? ch / (a.channels / a.groups) : 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        float y = 0.f, x = 0.f, z = 0.f;
        const int64_t n = (int64_t)set * R + i;
        if (slot[i] >= 0) {
            float b[8], c[8];
            load8<T>(static_cast<const T*>(a.b) + n * a.b_stride + group * S + ln * 8, packed, b);
            load8<T>(static_cast<const T*>(a.c) + n * a.c_stride + group * S + ln * 8, packed, c);
            x = widen<T>(static_cast<const T*>(a.x)[n * a.x_stride + ch]);
            if (a.z) z = widen<T>(static_cast<const T*>(a.z)[n * a.z_stride + ch]);
            float dt = widen<T>(static_cast<const T*>(a.dt)[n * a.dt_stride + ch]) + bias;
            if (a.softplus) dt = softplus_of(dt);
            const float dx = dt * x;
            Pack<float, 8> q;
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                q.v[s] = fmaf(ex2(dt * a2[s]), h[i][s], dx * b[s]);
                y = fmaf(q.v[s], c[s], y);
            }
            *reinterpret_cast<Pack<float, 8>*>(a.out_state + ((int64_t)slot[i] * a.channels + ch) * S + ln * 8) = q;
        }
#pragma unroll
        for (int m = LN / 2; m >= 1; m /= 2) y += __shfl_xor_sync(0xffffffffu, y, m);
        if (slot[i] >= 0 && ln == 0) {
            y = fmaf(skip, x, y);
            if (a.z) y *= silu_of(z);
            static_cast<T*>(a.out)[n * a.out_stride + ch] = round_to<T>(y);
        }
    }
}

template <typename T, int S, int R> cudaError_t launch(const ScanArgs& a, cudaStream_t stream)
{
    const uint64_t per = ((uint64_t)a.channels * (S / 8) + 31) / 32 * 32, sets = ((uint64_t)a.num_seqs + R - 1) / R;
    if (per * sets > 0xffffffffull - 128) return cudaErrorNotSupported;
    const uintptr_t rows = (uintptr_t)a.b | (uintptr_t)a.c | (uintptr_t)((a.b_stride | a.c_stride) * (int64_t)sizeof(T));
    return launch_kernel(selective_step_kernel<T, S, R>, (unsigned)((per * sets + 127) / 128), 128, 0, stream, 1, a, (uint32_t)per, rows % 16 == 0);
}

template <typename T, int S> cudaError_t launch_requests(const ScanArgs& a, cudaStream_t stream)
{
    // several requests per thread where that leaves every SM its 2,048 threads
    if ((int64_t)a.num_seqs * a.channels * (S / 8) >= 2ll * 148 * 2048) return launch<T, S, 2>(a, stream);
    return launch<T, S, 1>(a, stream);
}

template <typename T> cudaError_t launch_width(const ScanArgs& a, int states, cudaStream_t stream)
{
    switch (states) {
        case 8: return launch_requests<T, 8>(a, stream);
        case 16: return launch_requests<T, 16>(a, stream);
        case 32: return launch_requests<T, 32>(a, stream);
        case 64: return launch_requests<T, 64>(a, stream);
    }
    return cudaErrorNotSupported;
}

}  // namespace
}  // namespace scan

cudaError_t launch_scan_step(const ScanArgs& a, int io_dtype, int states, cudaStream_t stream)
{
    return io_dtype == GDN_BF16 ? scan::launch_width<__nv_bfloat16>(a, states, stream) : scan::launch_width<float>(a, states, stream);
}

}  // namespace gdn
