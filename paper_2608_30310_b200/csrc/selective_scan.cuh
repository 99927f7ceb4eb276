// Selective state space scan over packed prompts, one CTA per tile of channels of a request:
//
//     h = exp(dt a) h + dt x b,   y = c . h + d x,   out = y silu(z),   dt = softplus(dt + dt_bias)
//
// The state stays in registers from a request's first token to its last.  Four compute warps do the recurrence alone: a lane holds SS
// states of CC channels, LN = S / SS lanes share CC channels.  c . h is summed over the LN lanes TS rows at a time by exchanging
// halves, after which every lane holds some finished sums, so that n sums over LN lanes cost less than n exchanges.  Four helper
// warps run around them, in blocks of TB rows: they copy x, dt, z, b and c of the block after the next but one to shared memory, form dt
// and dt x of the next block (once for every row and channel), and finish the block before: skip, gate, rounding, store.  One
// barrier per block.
//
// Bound by its exponentials, not by memory: one result of the special-function unit per state and token, three more per channel and token.
// Eight hits (12,616 tokens, 4,096 channels, 16 states, bf16) take 301 us where the unit alone would take 215 and the memory 65; issue
// slots, unit and shared memory are 68-73 % busy.  One request of 1,638 tokens: 61 us (unit 28), one compute and one helper warp per
// scheduler, latency.  Everything in every warp, without roles, took 1,050 and 174 us.  32 rows a block: sixteen 334 us for eight hits.
#pragma once
#include <float.h>
#include "layers.cuh"

namespace gdn {
namespace scan {

// ex2.approx is low by 0.09 (arguments of 2^-9 and less) to 0.45 (2^-6) units of 2^-24 in the mean, which a state that decays slowly adds up
// over its whole memory: 120 units at 2^-10.  Added to the argument, a tenth of a unit leaves 40 at most (measured on a million arguments per
// octave); 2^kLift is still 1, so that a time step of zero changes nothing.
constexpr float kLift = 8.6e-9f;

// log(1 + e^x) = max(x, 0) + log1p(u), u = e^-|x| in (0, 1].  log1p(u) / u is the polynomial of degree eight nearest to it (least largest
// relative error, 3e-8, by Lawson's iteration); a logarithm of 1 + u would lose the small time steps that u << 1 stands for.
__device__ __forceinline__ F2 softplus_of(F2 x2)
{
    const float2 x = parts(x2);
    const F2 u = pair(ex2(-kLog2e * fabsf(x.x)), ex2(-kLog2e * fabsf(x.y)));
    F2 p = fma(u, both(0.005232692641f), both(-0.02950523219f));
    p = fma(u, p, both(0.07822594086f));
    p = fma(u, p, both(-0.136632448f));
    p = fma(u, p, both(0.191060062f));
    p = fma(u, p, both(-0.2484298196f));
    p = fma(u, p, both(0.3331909665f));
    p = fma(u, p, both(-0.4999949302f));
    p = fma(u, p, both(0.9999999694f));
    return fma(u, p, pair(fmaxf(x.x, 0.f), fmaxf(x.y, 0.f)));
}
__device__ __forceinline__ float softplus_of(float x)
{
    const float u = ex2(-kLog2e * fabsf(x));
    float p = fmaf(u, 0.005232692641f, -0.02950523219f);
    p = fmaf(u, p, 0.07822594086f);
    p = fmaf(u, p, -0.136632448f);
    p = fmaf(u, p, 0.191060062f);
    p = fmaf(u, p, -0.2484298196f);
    p = fmaf(u, p, 0.3331909665f);
    p = fmaf(u, p, -0.4999949302f);
    p = fmaf(u, p, 0.9999999694f);
    return fmaf(u, p, fmaxf(x, 0.f));
}

template <typename T, int N> __device__ __forceinline__ void load_values(const T* p, float (&v)[N])
{
    const Pack<T, N> q = *reinterpret_cast<const Pack<T, N>*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = widen<T>(q.v[i]);
}

constexpr int kCompute = 4, kHelpers = 4, kThreads = 32 * (kCompute + kHelpers), kRing = 4;

template <int S_, int SS_, int CC_, typename T> struct Form {
    static constexpr int S = S_, SS = SS_, CC = CC_;
    static constexpr int LN = S / SS, W = 32 * CC / LN, CT = kCompute * W;      // channels of a warp, of the CTA
    static constexpr int TS = LN / CC > 4 ? LN / CC : 4;     // rows of a reduction
    static constexpr int TB = 32;                             // rows of a block
    static constexpr int SUMS = TS * CC, MINE = SUMS / LN;   // sums of a reduction, and how many a lane ends up with
    static constexpr int PER = TB * CT / (32 * kHelpers);    // channels of a row that a helper has in hand at once
    static constexpr int VE = PER > 8 ? 8 : PER < 2 ? 2 : PER, ROWI = CT / VE, ITEMS = TB * ROWI, IPT = (ITEMS + 32 * kHelpers - 1) / (32 * kHelpers);
    // (dt, dt x) of two channels are 16 bytes; those of an item's channels 0 and 1, of all items of the row, come first (neighbouring lanes write
    // neighbouring 16 bytes), then, four words further on (a compute warp's channels are in different banks), those of channels 2 and 3, and
    // so on; y likewise by 16 or 8 bytes.
    static constexpr int PJ = 4 * ROWI + 4, PW = VE / 2 * PJ, PS = ROWI >= 8 ? PW : PW + (4 * ROWI - PW % 32 + 32) % 32;
    static constexpr int YV = VE < 4 ? VE : 4, YS = CT + 4;
    __host__ __device__ static constexpr int p_at(int ch) { return ch % VE / 2 * PJ + ch / VE * 4 + ch % 2 * 2; }
    __host__ __device__ static constexpr int y_at(int ch) { return (ch % VE / YV * ROWI + ch / VE) * YV + ch % YV; }
    static_assert(TB % TS == 0 && SUMS % LN == 0 && W * LN == 32 * CC && CT % VE == 0, "");
    static constexpr int BC = sizeof(T) == 2 ? 1 : 2;        // words of (b, c): packed bf16 halves, or one each
    struct Shared {
        alignas(16) T x[kRing][TB * CT], dt[kRing][TB * CT], z[kRing][TB * CT], b[kRing][TB * S], c[kRing][TB * S];
        alignas(16) float p[2][TB * PS];                 // (dt, dt x) of each row and channel
        alignas(16) uint32_t bc[2][BC][TB * S];
        alignas(16) float y[2][TB * YS];
        alignas(16) float bias[CT], skip[CT];
        int4 table[kSelfSort];
    };
};

// ALIGNED: rows of x, dt, z and out, and the channels of a group, come in whole vectors of VE values, rows of b and c in whole 8 bytes.
template <typename T, typename F, bool ALIGNED>
__global__ void __launch_bounds__(kThreads, F::SS * F::CC > 4 ? 2 : 3) selective_scan_kernel(const ScanArgs a, const uint32_t tiles, const bool ordered)
{
    constexpr int S = F::S, SS = F::SS, CC = F::CC, LN = F::LN, W = F::W, CT = F::CT, VE = F::VE, TB = F::TB, TS = F::TS;
    extern __shared__ __align__(16) unsigned char raw[];
    typename F::Shared& sh = *reinterpret_cast<typename F::Shared*>(raw);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

    wait_for_predecessor();
    const uint32_t place = blockIdx.x / tiles, tile = blockIdx.x - place * tiles;
    int4 req;                                                // (first row, end row, request)
    if (ordered) {
        sort_requests(a.cu, a.num_seqs, sh.table, warp, kCompute + kHelpers, lane);
        __syncthreads();
        req = sh.table[place];
    } else {
        req = make_int4(a.cu[place], a.cu[place + 1], (int)place, 0);
    }
    req.y = (int)min((int64_t)req.y, a.total_tokens);
    // tiles do not cross groups: b and c are one group's
    const int each = a.channels / a.groups, per = (each + CT - 1) / CT, group = tile / per, first = group * each + (tile - group * per) * CT;
    const int limit = (group + 1) * each;
    const int blocks = req.x < req.y ? (req.y - req.x + TB - 1) / TB : 0;

    if (warp >= kCompute) {
        const int id = threadIdx.x - 32 * kCompute;
        // dt_bias and d of the tile's channels
        for (int c = id; c < CT; c += 32 * kHelpers) {
            sh.bias[c] = a.dt_bias && first + c < limit ? a.dt_bias[first + c] : 0.f;
            sh.skip[c] = a.d && first + c < limit ? a.d[first + c] : 0.f;
        }
        // A helper's share of a block: ITEMS rows' pieces of VE channels (piece k is in row r0 + k RSTEP), and vectors of 8 bytes of b and c.  It
        // copies what it reads itself later: no barrier in between.
        constexpr int RSTEP = 32 * kHelpers / F::ROWI;
        static_assert(32 * kHelpers % F::ROWI == 0, "a helper keeps its channels");
        const int r0 = id / F::ROWI, ch = id % F::ROWI * VE;
        constexpr int V8 = 8 / sizeof(T), BCI = TB * S / V8, BPT = (BCI + 32 * kHelpers - 1) / (32 * kHelpers), BSTEP = 32 * kHelpers / (S / V8);
        static_assert(32 * kHelpers % (S / V8) == 0, "");
        const int b0 = id / (S / V8), bs = id % (S / V8) * V8;
        auto mine = [&](int k) { return F::ITEMS % (32 * kHelpers) == 0 || id + k * 32 * kHelpers < F::ITEMS; };
        auto mine_bc = [&](int k) { return BCI % (32 * kHelpers) == 0 || id + k * 32 * kHelpers < BCI; };
        const T* xp = static_cast<const T*>(a.x) + (int64_t)(req.x + r0) * a.x_stride + first + ch;      // of the block that is copied next
        const T* dp = static_cast<const T*>(a.dt) + (int64_t)(req.x + r0) * a.dt_stride + first + ch;
        const T* zp = static_cast<const T*>(a.z) + (int64_t)(req.x + r0) * a.z_stride + first + ch;
        const T* bp = static_cast<const T*>(a.b) + (int64_t)(req.x + b0) * a.b_stride + group * S + bs;
        const T* cp = static_cast<const T*>(a.c) + (int64_t)(req.x + b0) * a.c_stride + group * S + bs;
        T* op = static_cast<T*>(a.out) + (int64_t)(req.x + r0) * a.out_stride + first + ch;              // of the block that is finished next
        const bool real = first + ch < limit;
        auto copy = [&](const T* src, T* dst) {
            if (ALIGNED) {
                constexpr int B = VE * sizeof(T) > 16 ? 16 : VE * sizeof(T);
#pragma unroll
                for (int v = 0; v < VE; v += B / sizeof(T)) copy_async<B>(dst + v, src + v);
            } else {
#pragma unroll
                for (int v = 0; v < VE; ++v) dst[v] = first + ch + v < limit ? src[v] : round_to<T>(0.f);
            }
        };
        auto issue = [&](int block) {
            const int left = req.y - req.x - block * TB, slot = block % kRing;
#pragma unroll
            for (int k = 0; k < F::IPT; ++k) {
                if (mine(k) && real && r0 + k * RSTEP < left) {
                    const int at = (r0 + k * RSTEP) * CT + ch;
                    copy(xp + k * RSTEP * a.x_stride, &sh.x[slot][at]);
                    copy(dp + k * RSTEP * a.dt_stride, &sh.dt[slot][at]);
                    if (a.z) copy(zp + k * RSTEP * a.z_stride, &sh.z[slot][at]);
                }
            }
            xp += TB * a.x_stride; dp += TB * a.dt_stride; zp += TB * a.z_stride;
#pragma unroll
            for (int k = 0; k < BPT; ++k) {
                if (mine_bc(k) && b0 + k * BSTEP < left) {
                    const int at = (id + k * 32 * kHelpers) * V8;
                    const T *b = bp + k * BSTEP * a.b_stride, *c = cp + k * BSTEP * a.c_stride;
                    if (ALIGNED) {
                        copy_async<8>(&sh.b[slot][at], b);
                        copy_async<8>(&sh.c[slot][at], c);
                    } else {
#pragma unroll
                        for (int v = 0; v < V8; ++v) { sh.b[slot][at + v] = b[v]; sh.c[slot][at + v] = c[v]; }
                    }
                }
            }
            bp += TB * a.b_stride; cp += TB * a.c_stride;
        };
        auto commit = []() { asm volatile("cp.async.commit_group;" ::: "memory"); };
        // (dt, dt x) and (b, c) of a block.  Rows past the request's end become zeros, whatever lies there.  (The state does not take them in
        // either: with a = -inf a time step of zero is no number.)
        auto prepare = [&](int block) {
            const int slot = block % kRing, buf = block & 1, left = req.y - req.x - block * TB;
            Pack<T, V8> b[BPT], c[BPT];
#pragma unroll
            for (int k = 0; k < BPT; ++k) {
                if (!mine_bc(k)) break;
                b[k] = *reinterpret_cast<const Pack<T, V8>*>(&sh.b[slot][(id + k * 32 * kHelpers) * V8]);
                c[k] = *reinterpret_cast<const Pack<T, V8>*>(&sh.c[slot][(id + k * 32 * kHelpers) * V8]);
            }
#pragma unroll
            for (int k = 0; k < F::IPT; ++k) {
                if (!mine(k)) break;
                const int r = r0 + k * RSTEP, at = r * CT + ch;
                const Pack<T, VE> x = *reinterpret_cast<const Pack<T, VE>*>(&sh.x[slot][at]), dt = *reinterpret_cast<const Pack<T, VE>*>(&sh.dt[slot][at]);
#pragma unroll
                for (int v = 0; v < VE; v += 2) {
                    F2 d = add(pair_at(dt, v), *reinterpret_cast<const F2*>(&sh.bias[ch + v]));
                    if (a.softplus) d = softplus_of(d);
                    const float2 dv = parts(d), dx = parts(mul(d, pair_at(x, v)));
                    float4 q = make_float4(dv.x, dx.x, dv.y, dx.y);
                    if (r >= left) q = make_float4(0.f, 0.f, 0.f, 0.f);
                    *reinterpret_cast<float4*>(&sh.p[buf][r * F::PS + F::p_at(ch) + v / 2 * F::PJ]) = q;
                }
            }
#pragma unroll
            for (int k = 0; k < BPT; ++k) {
                if (!mine_bc(k)) break;
                const int at = (id + k * 32 * kHelpers) * V8;
                Pack<uint32_t, V8> lo, hi;
#pragma unroll
                for (int v = 0; v < V8; ++v) {
                    if constexpr (sizeof(T) == 2) lo.v[v] = (uint32_t)__bfloat16_as_ushort(b[k].v[v]) | (uint32_t)__bfloat16_as_ushort(c[k].v[v]) << 16;
                    else { lo.v[v] = __float_as_uint(b[k].v[v]); hi.v[v] = __float_as_uint(c[k].v[v]); }
                }
                if (b0 + k * BSTEP >= left) lo = hi = {};
                *reinterpret_cast<Pack<uint32_t, V8>*>(&sh.bc[buf][0][at]) = lo;
                if (sizeof(T) == 4) *reinterpret_cast<Pack<uint32_t, V8>*>(&sh.bc[buf][F::BC - 1][at]) = hi;
            }
        };
        auto finish = [&](int block) {
            const int slot = block % kRing, buf = block & 1, left = req.y - req.x - block * TB;
#pragma unroll
            for (int k = 0; k < F::IPT; ++k) {
                const int r = r0 + k * RSTEP, at = r * CT + ch;
                if (!mine(k) || !real || r >= left) break;
                const Pack<T, VE> x = *reinterpret_cast<const Pack<T, VE>*>(&sh.x[slot][at]);
                Pack<T, VE> z, o;
                if (a.z) z = *reinterpret_cast<const Pack<T, VE>*>(&sh.z[slot][at]);
#pragma unroll
                for (int u = 0; u < VE; u += F::YV) {
                    const Pack<float, F::YV> y = *reinterpret_cast<const Pack<float, F::YV>*>(&sh.y[buf][r * F::YS + F::y_at(ch) + u * F::ROWI]);
#pragma unroll
                    for (int v = 0; v < F::YV; v += 2) {
                        F2 w = fma(*reinterpret_cast<const F2*>(&sh.skip[ch + u + v]), pair_at(x, u + v), pair_at(y, v));
                        if (a.z) w = mul(w, silu_of(pair_at(z, u + v)));
                        const float2 f = parts(w);
                        o.v[u + v] = round_to<T>(f.x); o.v[u + v + 1] = round_to<T>(f.y);
                    }
                }
                T* dst = op + k * RSTEP * a.out_stride;
                if (ALIGNED) {
                    *reinterpret_cast<Pack<T, VE>*>(dst) = o;
                } else {
#pragma unroll
                    for (int v = 0; v < VE; ++v)
                        if (first + ch + v < limit) dst[v] = o.v[v];
                }
            }
            op += TB * a.out_stride;
        };
        for (int i = 0; i < kRing - 1; ++i) {
            if (i < blocks) issue(i);
            commit();
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 2) : "memory");
        asm volatile("bar.sync 1, %0;" ::"n"(32 * kHelpers) : "memory");     // (bias and skip)
        if (blocks > 0) prepare(0);
        __syncthreads();
        for (int i = 0; i < blocks; ++i) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 3) : "memory");
            if (i + 1 < blocks) prepare(i + 1);
            if (i > 0) finish(i - 1);
            if (i + kRing - 1 < blocks) issue(i + kRing - 1);                // (in the ring's place of block i - 1, which is done)
            commit();
            __syncthreads();
        }
        allow_successor();
        if (blocks > 0) finish(blocks - 1);
        return;
    }

    const int sub = lane / LN, ln = lane % LN, ch0 = warp * W + sub * CC;
    float h[CC][SS], a2[CC][SS];
    const int from = a.init_state ? slot_of(a.init_slots, req.z, a.num_init, a.status_word) : -1;
#pragma unroll
    for (int c = 0; c < CC; ++c) {
        const int ch = first + ch0 + c;
#pragma unroll
        for (int s = 0; s < SS; ++s) h[c][s] = a2[c][s] = 0.f;
        if (ch < limit) {
            load_values<float, SS>(a.a + (int64_t)ch * S + ln * SS, a2[c]);
            if (from >= 0) load_values<float, SS>(a.init_state + ((int64_t)from * a.channels + ch) * S + ln * SS, h[c]);
        }
#pragma unroll
        for (int s = 0; s < SS; ++s) {
            const float a = a2[c][s];                        // (one that is finite stays so: a time step of 0 leaves the state as it is)
            a2[c][s] *= kLog2e;
            if (isinf(a2[c][s]) && !isinf(a)) a2[c][s] = copysignf(FLT_MAX, a);
        }
    }
    __syncthreads();
    for (int block = 0; block < blocks; ++block) {
        const int buf = block & 1;
        const float* ps = &sh.p[buf][F::p_at(ch0)];
        const uint32_t *b0 = &sh.bc[buf][0][ln * SS], *b1 = &sh.bc[buf][F::BC - 1][ln * SS];
        float* ys = &sh.y[buf][F::y_at(ch0)];                // (CC channels are neighbours there)
        auto rows_of = [&](int t, float* sums, bool real) {                   // (not real: past the request's end, the state stays)
            float b[SS], c[SS], p[2 * CC];
            const Pack<uint32_t, SS> w = *reinterpret_cast<const Pack<uint32_t, SS>*>(b0 + t * S);
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int s = 0; s < SS; ++s) { b[s] = __uint_as_float(w.v[s] << 16); c[s] = __uint_as_float(w.v[s] & 0xffff0000u); }
            } else {
                const Pack<uint32_t, SS> w1 = *reinterpret_cast<const Pack<uint32_t, SS>*>(b1 + t * S);
#pragma unroll
                for (int s = 0; s < SS; ++s) { b[s] = __uint_as_float(w.v[s]); c[s] = __uint_as_float(w1.v[s]); }
            }
            load_values<float, 2 * CC>(ps + t * F::PS, p);
#pragma unroll
            for (int k = 0; k < CC; ++k) {
                const float dt = p[2 * k], dx = p[2 * k + 1];
                if constexpr (SS == 1) {
                    const float hn = fmaf(ex2(fmaf(dt, a2[k][0], kLift)), h[k][0], dx * b[0]);
                    h[k][0] = real ? hn : h[k][0];
                    sums[k] = hn * c[0];
                } else {
                    F2 acc;
#pragma unroll
                    for (int s = 0; s < SS; s += 2) {
                        const float2 e = parts(fma(pair(dt, dt), pair(a2[k][s], a2[k][s + 1]), both(kLift)));
                        const F2 hn = fma(pair(ex2(e.x), ex2(e.y)), pair(h[k][s], h[k][s + 1]), mul(pair(dx, dx), pair(b[s], b[s + 1])));
                        const float2 hv = parts(hn);
                        h[k][s] = real ? hv.x : h[k][s]; h[k][s + 1] = real ? hv.y : h[k][s + 1];
                        acc = s ? fma(hn, pair(c[s], c[s + 1]), acc) : mul(hn, pair(c[s], c[s + 1]));
                    }
                    const float2 r = parts(acc);
                    sums[k] = r.x + r.y;
                }
            }
        };
        // sum over LN lanes: each exchange halves what a lane is responsible for; lane ln ends with sums ln MINE ...
        auto reduce = [&](float (&sums)[F::SUMS]) {
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
        };
        auto store = [&](int t, const float (&sums)[F::SUMS]) {
#pragma unroll
            for (int i = 0; i < F::MINE; ++i) {
                const int j = ln * F::MINE + i;
                ys[(t + j / CC) * F::YS + j % CC] = sums[i];
            }
        };
        const int left = req.y - req.x - block * TB;
        if (left < TB) {                                     // the last block: no more rows than there are
#pragma unroll 1
            for (int t = 0; t < left; t += TS) {
                float sums[F::SUMS];
#pragma unroll
                for (int i = 0; i < TS; ++i) rows_of(t + i, &sums[i * CC], t + i < left);
                reduce(sums);
                store(t, sums);
            }
        } else {
            // the sums of TS rows are exchanged and stored while the next TS rows are computed: their loads come first, as the
            // compiler cannot move them across the stores
            float before[F::SUMS];
#pragma unroll
            for (int t = 0; t <= TB; t += TS) {
                float sums[F::SUMS];
                if (t < TB)
#pragma unroll
                    for (int i = 0; i < TS; ++i) rows_of(t + i, &sums[i * CC], true);
                if (t > 0) {
                    reduce(before);
                    store(t - TS, before);
                }
#pragma unroll
                for (int i = 0; i < F::SUMS; ++i) before[i] = sums[i];
            }
        }
        __syncthreads();
    }

    allow_successor();                                       // (earlier, the next call's CTAs crowd the SMs that are free already)
    const int to = a.out_state ? slot_of(a.out_slots, req.z, a.num_out, a.status_word) : -1;
    if (to < 0) return;
#pragma unroll
    for (int c = 0; c < CC; ++c) {
        const int ch = first + ch0 + c;
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
    const uint32_t tiles = (uint32_t)a.groups * ((each + F::CT - 1) / F::CT);
    const uint64_t grid = (uint64_t)a.num_seqs * tiles;
    if (grid > 0x7fffffffull) return cudaErrorNotSupported;
    const uintptr_t all = (uintptr_t)a.x | (uintptr_t)a.dt | (uintptr_t)a.z | (uintptr_t)a.out |
                          (uintptr_t)((a.x_stride | a.dt_stride | (a.z ? a.z_stride : 0) | a.out_stride) * (int64_t)sizeof(T));
    const uintptr_t bc = (uintptr_t)a.b | (uintptr_t)a.c | (uintptr_t)((a.b_stride | a.c_stride) * (int64_t)sizeof(T));
    const bool aligned = all % alignof(Pack<T, F::VE>) == 0 && bc % 8 == 0 && each % F::VE == 0;
    constexpr size_t smem = sizeof(typename F::Shared);
    static_assert(smem <= 227 * 1024, "what a CTA can have");
    // Longest first, up to the number of requests that a CTA orders itself, unless they are short: 64 of 64 tokens 140 us ordered, 121 not;
    // 16 of 33-700 tokens 181, 189; eight of 410-3,277 303, 429.
    const bool ordered = a.num_seqs > 1 && a.num_seqs <= kSelfSort && a.total_tokens >= 128ll * a.num_seqs;
    auto kernel = aligned ? selective_scan_kernel<T, F, true> : selective_scan_kernel<T, F, false>;
    if (smem > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    return launch_kernel<false>(kernel, (unsigned)grid, kThreads, smem, stream, 1, a, tiles, ordered);
}

// How many states a lane holds.  With fewer there are more warps, and each is sooner done with a row; with more, what is done once per lane
// and row (loads, sums) serves more of them.  By the states of the call per SM (requests x channels x states / 148); measured at 16
// states, bf16, us with one / two / four states a lane: one request of 1,638 tokens and 1,024 channels (111 per SM) 30 / 40 / 59; 2,048 channels
// (221) 49 / 40 / 59; 4,096 channels (443) 92 / 64 / 60; eight hits of 4,096 channels (3,542) 582 / 379 / 303.  fp32 reads twice the
// words of b and c per state, which two channels a lane share: four states of two channels, from more states on (4,096 channels 71 with
// two states a lane, 72 so; eight hits 445, 366; four states of one channel 398, two of two 375).  64 states are summed over 16 lanes, which two
// channels a lane halve (bf16, 4,096 channels 205 -> 168).  With 8 states that form's tiles do not fit the shared memory in fp32: two by two.
// The same borders at other numbers of states (700 tokens, bf16, us with one / two / the widest form): 8 states 110 per SM 16 / 22 / 36, 220 24 / 23 /
// 37, 320 33 / 32 / 37, 700 60 / 44 / 54, 1,400 107 / 86 / 87; 32 states 110 15 / 21 / 26, 220 23 / 21 / 26, 450 42 / 30 / 27, 700 59 / 41 / 42, 1,400 104 /
// 78 / 59; 64 states (two, the widest) 220 20 / 46, 450 30 / 47, 700 43 / 47, 1,400 82 / 74.  fp32: 8 states 700 66 / 62 / 80, 1,400 117 / 113 / 120; 32 states
// 450 52 / 34 / 44, 700 75 / 55 / 44, 1,400 139 / 100 / 88; 64 states 450 44 / 48, 700 64 / 47, 1,400 127 / 94.
template <typename T, int S> cudaError_t launch_states(const ScanArgs& a, cudaStream_t stream)
{
    const int64_t per_sm = (int64_t)a.num_seqs * a.channels * S / 148;
    if (S < 64 && per_sm <= 160) return launch_form<T, Form<S, S < 64 ? 1 : 2, 1, T>>(a, stream);
    if (per_sm <= (sizeof(T) == 2 && S < 64 ? 320 : 700)) return launch_form<T, Form<S, 2, 1, T>>(a, stream);
    constexpr bool half = sizeof(T) == 2;
    return launch_form<T, Form<S, !half && S == 8 ? 2 : 4, half && S < 64 ? 1 : 2, T>>(a, stream);
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
