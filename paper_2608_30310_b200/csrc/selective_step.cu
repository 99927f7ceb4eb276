// One token of the selective scan per request, from and to a state in memory.
//
// Bound by HBM: every state is read and written once (8 bytes), for one exponential and five flops.  A lane has four states of kChannels
// channels; S / 4 lanes share a channel, and the warp's accesses to the states are whole 512 bytes.
#include "selective_scan.cuh"

namespace gdn {
namespace scan {
namespace {

constexpr int kChannels = 2;           // of a lane: 256 requests of 4,096 channels and 16 states take 36 us with one, 29 with two, 34 with four

// A CTA of four warps has pieces of 4 * kChannels * 128 / S channels of one request.  PACKED: rows of b and c begin on four values.  GROUPS: there
// are several.  No branch stands among the loads, so that all of them are on their way at once: what a call leaves out (z, d, dt_bias)
// or a lane has not (channels past the last) is read from where something is, and not used.
template <typename T, int S, bool PACKED, bool GROUPS>
__global__ void __launch_bounds__(128) selective_step_kernel(const ScanArgs a, const uint32_t pieces)
{
    constexpr int LN = S / 4, ACROSS = 32 / LN, CC = kChannels, BC = GROUPS ? CC : 1;
    const int n = blockIdx.x / pieces, piece = blockIdx.x - n * pieces, lane = threadIdx.x % 32, ln = lane % LN;
    const int c0 = (piece * 4 + threadIdx.x / 32) * CC * ACROSS + lane / LN;     // and every ACROSS-th after it
    allow_successor();
    wait_for_predecessor();
    const int slot = slot_of(a.init_slots, n, min(a.num_init, a.num_out), a.status_word);
    if (slot < 0) return;
    const int64_t state = (int64_t)slot * a.channels * S + ln * 4;
    const T *xr = static_cast<const T*>(a.x) + n * a.x_stride, *dr = static_cast<const T*>(a.dt) + n * a.dt_stride;
    const T* zr = a.z ? static_cast<const T*>(a.z) + n * a.z_stride : xr;
    const T *br = static_cast<const T*>(a.b) + n * a.b_stride + ln * 4, *cr = static_cast<const T*>(a.c) + n * a.c_stride + ln * 4;
    const float *biases = a.dt_bias ? a.dt_bias : a.a, *skips = a.d ? a.d : a.a;
    const int each = a.channels / a.groups;
    Pack<float, 4> h[CC], d[CC];
    Pack<T, 4> b[BC], c[BC];
    T x[CC], dt[CC], z[CC];
    float bias[CC], skip[CC];
    auto load4 = [](const T* p) {
        Pack<T, 4> v;
        if (PACKED) v = *reinterpret_cast<const Pack<T, 4>*>(p);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i) v.v[i] = p[i];
        return v;
    };
#pragma unroll
    for (int k = 0; k < CC; ++k) {
        const int ch = min(c0 + k * ACROSS, a.channels - 1);
        h[k] = *reinterpret_cast<const Pack<float, 4>*>(a.init_state + state + (int64_t)ch * S);
        d[k] = *reinterpret_cast<const Pack<float, 4>*>(a.a + (int64_t)ch * S + ln * 4);
        x[k] = xr[ch];
        dt[k] = dr[ch];
        z[k] = zr[ch];
        bias[k] = biases[ch];
        skip[k] = skips[ch];
        if (GROUPS || k == 0) {
            const int g = GROUPS ? ch / each * S : 0;
            b[GROUPS ? k : 0] = load4(br + g);
            c[GROUPS ? k : 0] = load4(cr + g);
        }
    }
#pragma unroll
    for (int k = 0; k < CC; ++k) {
        const int ch = c0 + k * ACROSS;
        float step = widen<T>(dt[k]) + (a.dt_bias ? bias[k] : 0.f);
        if (a.softplus) step = softplus_of(step);
        const F2 arg = both(step * kLog2e), dx = both(step * widen<T>(x[k]));
        F2 acc;
#pragma unroll
        for (int s = 0; s < 4; s += 2) {
            const float2 e = parts(mul(arg, pair_at(d[k], s)));
            const F2 hn = fma(pair(ex2(e.x), ex2(e.y)), pair_at(h[k], s), mul(dx, pair_at(b[GROUPS ? k : 0], s)));
            acc = s ? fma(hn, pair_at(c[GROUPS ? k : 0], s), acc) : mul(hn, pair_at(c[GROUPS ? k : 0], s));
            const float2 v = parts(hn);
            h[k].v[s] = v.x; h[k].v[s + 1] = v.y;
        }
        if (ch < a.channels) *reinterpret_cast<Pack<float, 4>*>(a.out_state + state + (int64_t)ch * S) = h[k];
        const float2 sum = parts(acc);
        float y = sum.x + sum.y;
#pragma unroll
        for (int m = LN / 2; m >= 1; m /= 2) y += __shfl_xor_sync(0xffffffffu, y, m);
        if (a.d) y = fmaf(skip[k], widen<T>(x[k]), y);
        if (a.z) y *= silu_of(widen<T>(z[k]));
        if (ch < a.channels && ln == 0) (static_cast<T*>(a.out) + n * a.out_stride)[ch] = round_to<T>(y);
    }
}

template <typename T, int S> cudaError_t launch(const ScanArgs& a, cudaStream_t stream)
{
    constexpr int channels = 4 * kChannels * 128 / S;
    const uint64_t pieces = ((uint64_t)a.channels + channels - 1) / channels, grid = pieces * a.num_seqs;
    if (grid > 0x7fffffffull) return cudaErrorNotSupported;
    const uintptr_t bc = (uintptr_t)a.b | (uintptr_t)a.c | (uintptr_t)((a.b_stride | a.c_stride) * (int64_t)sizeof(T));
    const bool packed = bc % alignof(Pack<T, 4>) == 0;
    auto kernel = a.groups > 1 ? (packed ? selective_step_kernel<T, S, true, true> : selective_step_kernel<T, S, false, true>)
                               : (packed ? selective_step_kernel<T, S, true, false> : selective_step_kernel<T, S, false, false>);
    return launch_kernel(kernel, (unsigned)grid, 128, 0, stream, 1, a, (uint32_t)pieces);
}

template <typename T> cudaError_t launch_width(const ScanArgs& a, int states, cudaStream_t stream)
{
    switch (states) {
        case 8: return launch<T, 8>(a, stream);
        case 16: return launch<T, 16>(a, stream);
        case 32: return launch<T, 32>(a, stream);
        case 64: return launch<T, 64>(a, stream);
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
