// What the kernels of the recurrent layers (short convolution, selective scan) and of the cache's pages share.
#pragma once
#include "common.cuh"

namespace gdn {

// The io dtype's values as fp32, and back with one rounding (to nearest even).
template <typename T> __device__ __forceinline__ float widen(T x);
template <> __device__ __forceinline__ float widen<float>(float x) { return x; }
template <> __device__ __forceinline__ float widen<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T round_to(float x);
template <> __device__ __forceinline__ float round_to<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 round_to<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// N consecutive values, moved 16 bytes at a time (less where there are fewer).
template <typename T, int N> struct alignas(sizeof(T) * N % 16 == 0 ? 16 : sizeof(T) * N % 8 == 0 ? 8 : sizeof(T) * N % 4 == 0 ? 4 : 2) Pack {
    T v[N];
};

// 2^x and 1 / x by the special-function unit, each within two steps of fp32
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.4426950408889634f;
// x sigmoid(x)
__device__ __forceinline__ float silu_of(float x) { return x * rcp(1.f + ex2(-kLog2e * x)); }

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
__device__ __forceinline__ F2 add(F2 a, F2 b)
{
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 both(float a) { return pair(a, a); }
__device__ __forceinline__ F2 silu_of(F2 x)
{
    const float2 e = parts(mul(x, both(-kLog2e))), s = parts(add(pair(ex2(e.x), ex2(e.y)), both(1.f)));
    return mul(x, pair(rcp(s.x), rcp(s.y)));
}

// values v and v + 1 of a pack
template <typename T, int N> __device__ __forceinline__ F2 pair_at(const Pack<T, N>& p, int v) { return pair(widen<T>(p.v[v]), widen<T>(p.v[v + 1])); }

// asynchronous copies to shared memory
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
template <int B> __device__ __forceinline__ void copy_async(void* dst, const void* src)
{
    static_assert(B == 4 || B == 8 || B == 16, "");
    if (B == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(dst)), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_addr(dst)), "l"(src), "n"(B) : "memory");
}

// slots[n] (no list: n) where the pool has it, else -1; a slot past the pool's end is reported
__device__ __forceinline__ int slot_of(const int32_t* slots, int n, int num_slots, int32_t* status_word)
{
    const int s = slots ? slots[n] : n;
    if (s < num_slots) return s < 0 ? -1 : s;
    if (status_word) *status_word = GDN_ERR_BAD_INDEX;
    return -1;
}

// Arguments of the short convolution; all device pointers.
struct ConvArgs {
    const void *x, *weight, *bias, *init_state;
    void *out, *out_state;
    const int32_t *cu, *init_slots, *out_slots;
    int32_t* status_word;
    int64_t x_stride, out_stride, total_tokens;
    int32_t channels, num_seqs, num_init, num_out, silu;
};
cudaError_t launch_conv(const ConvArgs& a, int io_dtype, int width, bool step, cudaStream_t stream);

// Arguments of the selective scan; all device pointers.
struct ScanArgs {
    const void *x, *dt, *b, *c, *z;
    const float *a, *d, *dt_bias, *init_state;
    void* out;
    float* out_state;
    const int32_t *cu, *init_slots, *out_slots;
    int32_t* status_word;
    int64_t x_stride, dt_stride, b_stride, c_stride, z_stride, out_stride, total_tokens;
    int32_t channels, groups, num_seqs, num_init, num_out, softplus;
};
cudaError_t launch_scan(const ScanArgs& a, int io_dtype, int states, cudaStream_t stream);
cudaError_t launch_scan_step(const ScanArgs& a, int io_dtype, int states, cudaStream_t stream);

}  // namespace gdn
