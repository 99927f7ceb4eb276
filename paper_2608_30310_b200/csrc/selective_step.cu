// One token of the selective scan per request, from and to a state in memory.
//
// Bound by HBM: every state is read and written once (8 bytes), for one exponential and five flops; beside that, what a channel costs (time
// step, gate, addresses), so that a lane has eight states of a channel.  256 requests of 4,096 channels and 16 states: 28 us, 5.1 TB/s (26 us
// in a graph); 1,024 requests: 98 us, 5.8 TB/s.
#include "selective_scan.cuh"

namespace gdn {
namespace scan {
namespace {

// A lane has QUADS times four states, S / QUADS apart (its accesses and its neighbours' are whole sectors), of CC channels, every ACROSS-th.
template <int S_, int CC_, int QUADS_> struct StepForm {
    static constexpr int S = S_, CC = CC_, QUADS = QUADS_;
    static constexpr int LN = S / 4 / QUADS, ACROSS = 32 / LN, CHANNELS = 4 * CC * ACROSS;      // lanes of a channel; channels side by side; of a CTA
};

// A CTA of four warps has CHANNELS channels of one request.  PACKED: rows of b and c begin on four values.  GROUPS: there are several.  No
// branch stands among the loads, so that all of them are on their way at once: what a call leaves out (z, d, dt_bias) or a lane has not
// (channels past the last) is read from where something is, and not used.
template <typename T, typename F, bool PACKED, bool GROUPS>
__global__ void __launch_bounds__(128) selective_step_kernel(const ScanArgs a)
{
    constexpr int S = F::S, LN = F::LN, ACROSS = F::ACROSS, CC = F::CC, Q = F::QUADS, BC = GROUPS ? CC : 1;
    const int n = blockIdx.x, lane = threadIdx.x % 32, ln = lane % LN;
    const int c0 = blockIdx.y * F::CHANNELS + threadIdx.x / 32 * CC * ACROSS + lane / LN;
    allow_successor();
    wait_for_predecessor();
    const int slot = slot_of(a.init_slots, n, min(a.num_init, a.num_out), a.status_word);
    if (slot < 0) return;
    const float* in = a.init_state + (int64_t)slot * a.channels * S + ln * 4;
    float* keep = a.out_state + (int64_t)slot * a.channels * S + ln * 4;
    const T *xr = static_cast<const T*>(a.x) + n * a.x_stride, *dr = static_cast<const T*>(a.dt) + n * a.dt_stride;
    const T* zr = a.z ? static_cast<const T*>(a.z) + n * a.z_stride : xr;
    const T *br = static_cast<const T*>(a.b) + n * a.b_stride + ln * 4, *cr = static_cast<const T*>(a.c) + n * a.c_stride + ln * 4;
    const float *biases = a.dt_bias ? a.dt_bias : a.a, *skips = a.d ? a.d : a.a;
    const int each = a.channels / a.groups;
    Pack<float, 4> h[CC][Q], d[CC][Q];
    Pack<T, 4> b[BC][Q], c[BC][Q];
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
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            h[k][q] = *reinterpret_cast<const Pack<float, 4>*>(in + (int64_t)ch * S + q * (S / Q));
            d[k][q] = *reinterpret_cast<const Pack<float, 4>*>(a.a + (int64_t)ch * S + ln * 4 + q * (S / Q));
            if (GROUPS || k == 0) {
                const int g = (GROUPS ? ch / each * S : 0) + q * (S / Q);
                b[GROUPS ? k : 0][q] = load4(br + g);
                c[GROUPS ? k : 0][q] = load4(cr + g);
            }
        }
        x[k] = xr[ch];
        dt[k] = dr[ch];
        z[k] = zr[ch];
        bias[k] = biases[ch];
        skip[k] = skips[ch];
    }
#pragma unroll
    for (int k = 0; k < CC; ++k) {
        const int ch = c0 + k * ACROSS;
        const bool real = ch < a.channels;
        float step = widen<T>(dt[k]) + (a.dt_bias ? bias[k] : 0.f);
        if (a.softplus) step = softplus_of(step);
        const F2 arg = both(step * kLog2e), dx = both(step * widen<T>(x[k]));
        F2 acc = both(0.f);
#pragma unroll
        for (int q = 0; q < Q; ++q) {
#pragma unroll
            for (int s = 0; s < 4; s += 2) {
                const float2 e = parts(fma(arg, pair_at(d[k][q], s), both(kLift)));
                const F2 hn = fma(pair(ex2(e.x), ex2(e.y)), pair_at(h[k][q], s), mul(dx, pair_at(b[GROUPS ? k : 0][q], s)));
                acc = fma(hn, pair_at(c[GROUPS ? k : 0][q], s), acc);
                const float2 v = parts(hn);
                h[k][q].v[s] = v.x; h[k][q].v[s + 1] = v.y;
            }
            if (real) *reinterpret_cast<Pack<float, 4>*>(keep + (int64_t)ch * S + q * (S / Q)) = h[k][q];
        }
        const float2 sum = parts(acc);
        float y = sum.x + sum.y;
#pragma unroll
        for (int m = LN / 2; m >= 1; m /= 2) y += __shfl_xor_sync(0xffffffffu, y, m);
        if (a.d) y = fmaf(skip[k], widen<T>(x[k]), y);
        if (a.z) y *= silu_of(widen<T>(z[k]));
        if (real && ln == 0) (static_cast<T*>(a.out) + n * a.out_stride)[ch] = round_to<T>(y);
    }
}

template <typename T, int S> cudaError_t launch(const ScanArgs& a, cudaStream_t stream)
{
    // (256 requests of 4,096 channels and 16 states, us by channels x quads of a lane: 1 x 2 32.3, 2 x 1 29.2, 2 x 2 27.1, 3 x 2 30.1, 4 x 2 29.6; 22.1 at the copy rate)
    using F = StepForm<S, 2, S == 8 ? 1 : 2>;
    const int64_t pieces = ((int64_t)a.channels + F::CHANNELS - 1) / F::CHANNELS;
    if (pieces > 65535) return cudaErrorNotSupported;
    const uintptr_t bc = (uintptr_t)a.b | (uintptr_t)a.c | (uintptr_t)((a.b_stride | a.c_stride) * (int64_t)sizeof(T));
    const bool packed = bc % alignof(Pack<T, 4>) == 0;
    auto kernel = a.groups > 1 ? (packed ? selective_step_kernel<T, F, true, true> : selective_step_kernel<T, F, false, true>)
                               : (packed ? selective_step_kernel<T, F, true, false> : selective_step_kernel<T, F, false, false>);
    return launch_kernel(kernel, dim3((unsigned)a.num_seqs, (unsigned)pieces), 128, 0, stream, 1, a);
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
