// Selective state space scan over packed prompts, one warp per tile of channels of a request:
//
//     h = exp(dt a) h + dt x b,   y = c . h + d x,   out = y silu(z),   dt = softplus(dt + dt_bias)
//
// The state stays in registers from a request's first token to its last.  A lane holds SS states of CC channels (EPL = SS CC), LN =
// S / SS lanes share CC channels, a warp has W = 32 CC / LN of them.  It goes through the request in blocks of TB rows:
//   1. lane = (row, VE channels): softplus(dt + dt_bias) and dt x, once for every (row, channel), into shared memory;
//   2. lane = (channels, states): the recurrence, row by row.  c . h is summed over the LN lanes TS rows at a time by exchanging
//      halves, after which every lane holds some finished sums, so that n sums over LN lanes cost less than n exchanges;
//   3. lane = (row, VE channels) again: skip, gate, rounding, store.
// x, dt, z of the next block are loaded into registers, b and c copied to shared memory, under the current one.  Warps share nothing.
#pragma once
#include "layers.cuh"

namespace gdn {
namespace scan {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// log(1 + e^x).  log1p(u) = 2 atanh(u / (2 + u)): the odd series in s = u / (2 + u) <= 1/3, cut where the next term is below half a
// step of fp32; a logarithm of 1 + u itself would lose the small time steps that e^x << 1 stands for.
__device__ __forceinline__ float softplus_of(float x)
{
    const float u = __expf(-fabsf(x)), s = __fdividef(u, 2.f + u), q = s * s;
    float p = fmaf(q, 2.f / 15.f, 2.f / 13.f);
    p = fmaf(q, p, 2.f / 11.f);
    p = fmaf(q, p, 2.f / 9.f);
    p = fmaf(q, p, 2.f / 7.f);
    p = fmaf(q, p, 2.f / 5.f);
    p = fmaf(q, p, 2.f / 3.f);
    p = fmaf(q, p, 2.f);
    return fmaf(s, p, fmaxf(x, 0.f));
}

// ---- pairs of fp32 values in one register pair (add, multiply, fma on both at once)
struct F2 { unsigned long long v; };
__device__ __forceinline__ F2 pair(float a, float b)
{
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 parts(F2 a)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
    return r;
}
__device__ __forceinline__ F2 mul(F2 a, F2 b)
{
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c)
{
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// asynchronous copies to shared memory; a size of 0 fills with zeros
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
template <int B> __device__ __forceinline__ void copy_async(void* dst, const void* src, bool there)
{
    if (B == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_addr(dst)), "l"(src), "r"(there ? 4 : 0) : "memory");
}

template <typename T, int N> __device__ __forceinline__ void load_values(const T* p, float (&v)[N])
{
    const Pack<T, N> q = *reinterpret_cast<const Pack<T, N>*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = widen<T>(q.v[i]);
}

template <int S_, int SS_, int CC_, typename T> struct Form {
    static constexpr int S = S_, SS = SS_, CC = CC_;
    static constexpr int LN = S / SS, W = 32 * CC / LN;
    static constexpr int VE = W < 8 ? W : 8;                 // channels of an item
    static constexpr int TB = 32 * VE / W;                   // rows of a block: one item per lane
    static constexpr int TS = LN / CC > 4 ? LN / CC : (TB < 4 ? TB : 4);
    static constexpr int SUMS = TS * CC, MINE = SUMS / LN;   // sums of a reduction, and how many a lane ends up with
    static_assert(TB % TS == 0 && SUMS % LN == 0 && W * LN == 32 * CC, "");
    static constexpr int PS = 2 * W + 4, YS = W + 4;         // row strides: the lanes of an item-wise access hit different banks
    struct Shared {
        alignas(16) T b[2][TB * S], c[2][TB * S];
        alignas(16) float p[TB * PS];                        // (dt, dt x) of each row and channel
        alignas(16) float y[TB * YS];
    };
};

constexpr int kWarps = 4;

// ALIGNED: rows of x, dt, z and out, and the channels of a group, come in whole vectors of VE values.
template <typename T, typename F, bool ALIGNED>
__global__ void __launch_bounds__(32 * kWarps) selective_scan_kernel(const ScanArgs a, const uint32_t tiles, const uint32_t ctas)
{
    constexpr int S = F::S, SS = F::SS, CC = F::CC, LN = F::LN, W = F::W, VE = F::VE, TB = F::TB, TS = F::TS;
    extern __shared__ __align__(16) unsigned char raw[];
    __shared__ int4 table[kSelfSort];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    typename F::Shared& sh = reinterpret_cast<typename F::Shared*>(raw)[warp];

    allow_successor();
    wait_for_predecessor();
    const uint32_t place = blockIdx.x / ctas, tile = (blockIdx.x - place * ctas) * kWarps + warp;
    int4 req;                                                // (first row, end row, request)
    if (a.num_seqs > 1 && a.num_seqs <= kSelfSort) {         // longest first; more requests than that fill the GPU in any order
        sort_requests(a.cu, a.num_seqs, table, warp, kWarps, lane);
        __syncthreads();
        req = table[place];
    } else {
        req = make_int4(a.cu[place], a.cu[place + 1], (int)place, 0);
    }
    if (tile >= tiles) return;
    req.y = (int)min((int64_t)req.y, a.total_tokens);
    // tiles do not cross groups: b and c are one group's
    const int each = a.channels / a.groups, per = (each + W - 1) / W, group = tile / per, first = group * each + (tile - group * per) * W;
    const int limit = (group + 1) * each;

    // lane = (channels, states)
    const int sub = lane / LN, ln = lane % LN;
    float h[CC][SS], a2[CC][SS];
    const int from = a.init_state ? slot_of(a.init_slots, req.z, a.num_init, a.status_word) : -1;
#pragma unroll
    for (int c = 0; c < CC; ++c) {
        const int ch = first + sub * CC + c;
#pragma unroll
        for (int s = 0; s < SS; ++s) h[c][s] = a2[c][s] = 0.f;
        if (ch < limit) {
            load_values<float, SS>(a.a + (int64_t)ch * S + ln * SS, a2[c]);
            if (from >= 0) load_values<float, SS>(a.init_state + ((int64_t)from * a.channels + ch) * S + ln * SS, h[c]);
        }
#pragma unroll
        for (int s = 0; s < SS; ++s) a2[c][s] *= kLog2e;
    }

    // lane = (row, VE channels)
    const int irow = lane / (W / VE), ich = (lane % (W / VE)) * VE, ch0 = first + ich;
    float bias[VE], skip[VE];
#pragma unroll
    for (int v = 0; v < VE; ++v) {
        bias[v] = a.dt_bias && ch0 + v < limit ? a.dt_bias[ch0 + v] : 0.f;
        skip[v] = a.d && ch0 + v < limit ? a.d[ch0 + v] : 0.f;
    }
    Pack<T, VE> xn, dn, zn;
    auto fetch = [&](const void* base, int64_t stride, int t, Pack<T, VE>& p) {
        const T* src = static_cast<const T*>(base) + (int64_t)(t + irow) * stride + ch0;
        if (ALIGNED && t + irow < req.y && ch0 < limit) {
            p = *reinterpret_cast<const Pack<T, VE>*>(src);
        } else {
#pragma unroll
            for (int v = 0; v < VE; ++v) p.v[v] = !ALIGNED && t + irow < req.y && ch0 + v < limit ? src[v] : round_to<T>(0.f);
        }
    };
    // rows past the request's end are zeros: whatever lies there, the state and the sums of the rows before do not see it
    auto stage = [&](const void* base, int64_t stride, int t, T* dst) {
        const T* src = static_cast<const T*>(base) + (int64_t)group * S;
        const uintptr_t al = (uintptr_t)src | (uintptr_t)(stride * (int64_t)sizeof(T));
        constexpr int V16 = 16 / sizeof(T), V4 = 4 / sizeof(T);
        if ((al & 15) == 0) {
            for (int i = lane; i < TB * S / V16; i += 32) {
                const int r = i / (S / V16), s = i % (S / V16) * V16;
                const bool there = t + r < req.y;
                copy_async<16>(dst + r * S + s, there ? src + (int64_t)(t + r) * stride + s : src, there);
            }
        } else if ((al & 3) == 0) {
            for (int i = lane; i < TB * S / V4; i += 32) {
                const int r = i / (S / V4), s = i % (S / V4) * V4;
                const bool there = t + r < req.y;
                copy_async<4>(dst + r * S + s, there ? src + (int64_t)(t + r) * stride + s : src, there);
            }
        } else {
            for (int i = lane; i < TB * S; i += 32) {
                const int r = i / S, s = i % S;
                dst[i] = t + r < req.y ? src[(int64_t)(t + r) * stride + s] : round_to<T>(0.f);
            }
        }
    };
    auto fetch_all = [&](int t, int buf) {
        fetch(a.x, a.x_stride, t, xn);
        fetch(a.dt, a.dt_stride, t, dn);
        if (a.z) fetch(a.z, a.z_stride, t, zn);
        stage(a.b, a.b_stride, t, sh.b[buf]);
        stage(a.c, a.c_stride, t, sh.c[buf]);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };

    if (req.x < req.y) fetch_all(req.x, 0);
    int buf = 0;
    for (int t0 = req.x; t0 < req.y; t0 += TB, buf ^= 1) {
        const Pack<T, VE> x = xn, z = zn;
        const bool there = t0 + irow < req.y;
#pragma unroll
        for (int v = 0; v < VE; ++v) {
            float dt = widen<T>(dn.v[v]) + bias[v];
            if (a.softplus) dt = softplus_of(dt);
            if (!there) dt = 0.f;
            *reinterpret_cast<float2*>(&sh.p[irow * F::PS + 2 * (ich + v)]) = make_float2(dt, dt * widen<T>(x.v[v]));
        }
        if (t0 + TB < req.y) {
            fetch_all(t0 + TB, buf ^ 1);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        __syncwarp();

#pragma unroll 1
        for (int t = 0; t < TB; t += TS) {
            float sums[F::SUMS];
#pragma unroll
            for (int i = 0; i < TS; ++i) {
                float b[SS], c[SS], p[2 * CC];
                load_values<T, SS>(&sh.b[buf][(t + i) * S + ln * SS], b);
                load_values<T, SS>(&sh.c[buf][(t + i) * S + ln * SS], c);
                load_values<float, 2 * CC>(&sh.p[(t + i) * F::PS + sub * CC * 2], p);
#pragma unroll
                for (int k = 0; k < CC; ++k) {
                    const float dt = p[2 * k], dx = p[2 * k + 1];
                    if constexpr (SS == 1) {
                        h[k][0] = fmaf(ex2(dt * a2[k][0]), h[k][0], dx * b[0]);
                        sums[i * CC + k] = h[k][0] * c[0];
                    } else {
                        F2 acc;
#pragma unroll
                        for (int s = 0; s < SS; s += 2) {
                            const float2 e = parts(mul(pair(dt, dt), pair(a2[k][s], a2[k][s + 1])));
                            const F2 hn = fma(pair(ex2(e.x), ex2(e.y)), pair(h[k][s], h[k][s + 1]), mul(pair(dx, dx), pair(b[s], b[s + 1])));
                            const float2 hv = parts(hn);
                            h[k][s] = hv.x; h[k][s + 1] = hv.y;
                            acc = s ? fma(hn, pair(c[s], c[s + 1]), acc) : mul(hn, pair(c[s], c[s + 1]));
                        }
                        const float2 r = parts(acc);
                        sums[i * CC + k] = r.x + r.y;
                    }
                }
            }
            // sum over LN lanes: each exchange halves what a lane is responsible for; lane ln ends with sums ln MINE ...
#pragma unroll
            for (int m = LN / 2, n = F::SUMS / 2; m >= 1; m /= 2, n /= 2) {
                const bool up = ln & m;
#pragma unroll
                for (int i = 0; i < F::SUMS / 2; ++i) {
                    if (i < n) {
                        const float other = __shfl_xor_sync(0xffffffffu, up ? sums[i] : sums[i + n], m);
                        sums[i] = (up ? sums[i + n] : sums[i]) + other;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < F::MINE; ++i) {
                const int j = ln * F::MINE + i;
                sh.y[(t + j / CC) * F::YS + sub * CC + j % CC] = sums[i];
            }
        }
        __syncwarp();

        Pack<T, VE> o;
#pragma unroll
        for (int v = 0; v < VE; ++v) {
            float y = fmaf(skip[v], widen<T>(x.v[v]), sh.y[irow * F::YS + ich + v]);
            if (a.z) y *= silu_of(widen<T>(z.v[v]));
            o.v[v] = round_to<T>(y);
        }
        T* dst = static_cast<T*>(a.out) + (int64_t)(t0 + irow) * a.out_stride + ch0;
        if (ALIGNED) {
            if (there && ch0 < limit) *reinterpret_cast<Pack<T, VE>*>(dst) = o;
        } else {
#pragma unroll
            for (int v = 0; v < VE; ++v)
                if (there && ch0 + v < limit) dst[v] = o.v[v];
        }
    }

    const int to = a.out_state ? slot_of(a.out_slots, req.z, a.num_out, a.status_word) : -1;
    if (to < 0) return;
#pragma unroll
    for (int c = 0; c < CC; ++c) {
        const int ch = first + sub * CC + c;
        if (ch >= limit) continue;
        Pack<float, SS> q;
#pragma unroll
        for (int s = 0; s < SS; ++s) q.v[s] = h[c][s];
        *reinterpret_cast<Pack<float, SS>*>(a.out_state + ((int64_t)to * a.channels + ch) * S + ln * SS) = q;
    }
}

template <typename T, typename F> cudaError_t launch_form(const ScanArgs& a, cudaStream_t stream)
{
    const int each = a.channels / a.groups;
    const uint32_t tiles = (uint32_t)a.groups * ((each + F::W - 1) / F::W), ctas = (tiles + kWarps - 1) / kWarps;
    const uint64_t grid = (uint64_t)a.num_seqs * ctas;
    if (grid > 0x7fffffffull) return cudaErrorNotSupported;
    const uintptr_t all = (uintptr_t)a.x | (uintptr_t)a.dt | (uintptr_t)a.z | (uintptr_t)a.out |
                          (uintptr_t)((a.x_stride | a.dt_stride | (a.z ? a.z_stride : 0) | a.out_stride) * (int64_t)sizeof(T));
    const bool aligned = all % alignof(Pack<T, F::VE>) == 0 && each % F::VE == 0;
    constexpr size_t smem = kWarps * sizeof(typename F::Shared);
    auto kernel = aligned ? selective_scan_kernel<T, F, true> : selective_scan_kernel<T, F, false>;
    if (smem > 40 * 1024) {                                  // (48 KB with the table of requests go without asking)
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    return launch_kernel(kernel, (unsigned)grid, 32 * kWarps, smem, stream, 1, a, tiles, ctas);
}

// Lanes per state: the fewer states a lane holds the more warps there are, and the more a state costs.
template <typename T, int S> cudaError_t launch_states(const ScanArgs& a, cudaStream_t stream)
{
    const int64_t all = (int64_t)a.num_seqs * a.channels * S;
    if (all > 148 * 4 * 32 * 16) return launch_form<T, Form<S, 4, 4, T>>(a, stream);
    if (all > 148 * 4 * 32) return launch_form<T, Form<S, 2, 2, T>>(a, stream);
    return launch_form<T, Form<S, S == 64 ? 2 : 1, 1, T>>(a, stream);
}

template <typename T> cudaError_t launch_type(const ScanArgs& a, int states, cudaStream_t stream)
{
    switch (states) {
        case 8: return launch_states<T, 8>(a, stream);
        case 16: return launch_states<T, 16>(a, stream);
        case 32: return launch_states<T, 32>(a, stream);
        case 64: return launch_states<T, 64>(a, stream);
    }
    return cudaErrorNotSupported;
}

}  // namespace scan
}  // namespace gdn
