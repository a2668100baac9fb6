// Logits of the policy that tokens are drawn from: penalties for repeated tokens, bias, temperature and grammar mask, with
// the log-sum-exp and the log-prob of a chosen token of the adjusted row in the same pass; and the gradient back through it.
//
//   u = z;  token in the row's history: u = u > 0 ? u / repetition : u repetition
//   u -= frequency n + presence [n > 0]      (n: how often the token is in the history behind the prompt)
//   u = (u + bias) / temperature;  not allowed: u = -inf
//   lse = log sum_j exp u_j,  logp = u_y - lse
//   dz = du / temperature * (in the history: z > 0 ? 1 / repetition : repetition), 0 where not allowed
//
// A row is cut into parts, a workgroup each, whose entries are in flight while the row's history is read.  The history
// becomes one number per entry of the part in LDS: what penalties add to the logit (forward) or what its gradient is
// multiplied with (backward).  The part is then folded from registers at one addition or product an entry: a test per
// entry for a token of the history, with its two divisions behind it, costs more than the exponential (scoring of 8,192 x
// 50,001 bfloat16 with it 1,050 us).  Maximum and sum of exp are taken before the temperature, which then is part of the
// exponent's scale.  All arithmetic is fp32; what is stored in bfloat16 is rounded once, and lse and logp are those of the
// fp32 values.  The kernels are bound by memory.
#include "a3po_common.h"
#include "a3po_launch.h"

namespace a3po {
namespace {

constexpr int kThreads = kAdjustThreads;
constexpr uint32_t kSeen = 0x80000000u;
constexpr float kInf = __builtin_huge_valf(), kLowest = -3.402823466e38f;

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2), aligned(2)));
typedef int32_t i32x4_any __attribute__((ext_vector_type(4), aligned(4)));

struct RowPolicy {
    float repetition, frequency, presence, inv_temperature;
    int64_t start;
    int len, prompt;
};

// what the row's arrays say; histories are cut to the tokens there are, absent arrays are neutral
__device__ __forceinline__ RowPolicy row_policy(const AdjustArgs &a, int64_t t)
{
    RowPolicy p;
    p.repetition = a.repetition ? a.repetition[t] : 1.0f;
    p.frequency = a.frequency ? a.frequency[t] : 0.0f;
    p.presence = a.presence ? a.presence[t] : 0.0f;
    p.inv_temperature = a.temperature ? 1.0f / a.temperature[t] : 1.0f;
    p.start = 0;
    p.len = p.prompt = 0;
    if (a.history) {
        const int64_t start = a.hist_start[t], len = a.hist_len[t];
        if (start >= 0 && start < a.history_tokens && len > 0) {
            p.start = start;
            p.len = (int)min(len, a.history_tokens - start);
        }
        p.prompt = a.prompt_len ? a.prompt_len[t] : 0;
    }
    return p;
}

// f(place in the history, place in the part) for every token of the row's history that lies in [first, first + span); four
// tokens a load, four loads of a thread in flight
template <typename F>
__device__ __forceinline__ void each_token(const AdjustArgs &a, const RowPolicy &p, int64_t first, int span, F f)
{
    const int32_t *h = a.history + p.start;
    const int base = (int)first;
    auto one = [&](int i, int32_t id) {
        // (ids and places are below 2^31: the difference of the bit patterns is below span only for those of the part)
        const uint32_t at = (uint32_t)id - (uint32_t)base;
        if (id >= 0 && at < (uint32_t)span) f(i, (int)at);
    };
    constexpr uint32_t kLoads = 4, kRound = kThreads * 4 * kLoads;
    const uint32_t len = (uint32_t)p.len, lane = threadIdx.x;
    uint32_t i = 0;  // (unsigned: lengths end below 2^31, the places tried beyond them below 2^32)
    for (; len - i >= kRound; i += kRound) {
        i32x4_any v[kLoads];
#pragma unroll
        for (uint32_t j = 0; j < kLoads; ++j) v[j] = *reinterpret_cast<const i32x4_any *>(h + i + (j * kThreads + lane) * 4);
#pragma unroll
        for (uint32_t j = 0; j < kLoads; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) one((int)(i + (j * kThreads + lane) * 4) + k, v[j][k]);
    }
    for (; i < len; i += kThreads * kLoads) {
        int32_t v[kLoads];
#pragma unroll
        for (uint32_t j = 0; j < kLoads; ++j) {
            const uint32_t at = i + j * kThreads + lane;
            v[j] = at < len ? h[at] : -1;
        }
#pragma unroll
        for (uint32_t j = 0; j < kLoads; ++j) one((int)(i + j * kThreads + lane), v[j]);
    }
}

__device__ __forceinline__ void fill(float *to, int span, float v)
{
    const int vecs = (span + 3) / 4;  // (parts end at multiples of 512: the last vector is there)
    for (int i = threadIdx.x; i < vecs; i += kThreads) reinterpret_cast<float4 *>(to)[i] = make_float4(v, v, v, v);
}

// What the penalties add to the entries [first, first + span) of row t, into `delta`.  Occurrences are counted there first
// (integers: the order of the additions does not matter; the top bit stands for those in the prompt); whoever adds the
// first one of a token notes its place, and each place noted is then turned into a difference.
template <typename ZT>
__device__ __forceinline__ void penalties(const AdjustArgs &a, const RowPolicy &p, const char *row, int64_t first, int span,
                                          float *delta, uint16_t *places, int *noted)
{
    uint32_t *cnt = reinterpret_cast<uint32_t *>(delta);
    __syncthreads();  // (the part before this one is done with the array)
    fill(delta, span, 0.0f);
    if (threadIdx.x == 0) *noted = 0;
    __syncthreads();
    each_token(a, p, first, span, [&](int i, int at) {
        const uint32_t old = i < p.prompt ? atomicOr(&cnt[at], kSeen) : atomicAdd(&cnt[at], 1u);
        if (old == 0) places[atomicAdd(noted, 1)] = (uint16_t)at;
    });
    __syncthreads();
    const int n = *noted;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int at = places[i];
        const uint32_t out = cnt[at] & ~kSeen;
        const float z = load_elem<ZT>(row, at);
        float u = z > 0.0f ? z / p.repetition : z * p.repetition;
        if (out) u -= fmaf(p.frequency, (float)out, p.presence);
        delta[at] = fabsf(z) == kInf ? 0.0f : u - z;  // (an infinite logit stays what it is)
    }
    __syncthreads();
}

__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float scale)
{
    MaxSum o;
    o.m = fmaxf(a.m, b.m);
    o.s = a.s * exp2_hw((a.m - o.m) * scale) + b.s * exp2_hw((b.m - o.m) * scale);
    return o;
}

__device__ __forceinline__ MaxSum wave_join(MaxSum v, float scale)
{
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) {
        MaxSum o;
        o.m = __shfl_xor(v.m, off, kWave);
        o.s = __shfl_xor(v.s, off, kWave);
        v = join(v, o, scale);
    }
    return v;
}

template <typename UT, int EPV>
__device__ __forceinline__ void store_out(char *p, const float *f)
{
    if constexpr (UT::kBytes * EPV >= 16) {
#pragma unroll
        for (int k = 0; k < EPV; k += UT::kPerVec) {
            const uint4 v = pack<UT>(f + k);
            const u32x4_t t = {v.x, v.y, v.z, v.w};
            __builtin_nontemporal_store(t, reinterpret_cast<u32x4_elem_t *>(p + k * UT::kBytes));
        }
    } else {
        const u32x2_t t = {pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])};
        __builtin_nontemporal_store(t, reinterpret_cast<u32x2_t *>(p));
    }
}

template <typename UT, int EPV>
__device__ __forceinline__ void load_in(const char *p, float *f)
{
    if constexpr (UT::kBytes * EPV >= 16) {
#pragma unroll
        for (int k = 0; k < EPV; k += UT::kPerVec) unpack<UT>(row_load<true>(p + k * UT::kBytes), f + k);
    } else {
        const u32x2_t t = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t *>(p));
        f[0] = __uint_as_float(t.x << 16), f[1] = __uint_as_float(t.x & 0xFFFF0000u);
        f[2] = __uint_as_float(t.y << 16), f[3] = __uint_as_float(t.y & 0xFFFF0000u);
    }
}

// EPV consecutive floats: from LDS (16-byte aligned), from memory (at any float)
template <int EPV>
__device__ __forceinline__ void load_lds(const float *p, float *f)
{
#pragma unroll
    for (int k = 0; k < EPV; k += 4) {
        const float4 w = *reinterpret_cast<const float4 *>(p + k);
        f[k] = w.x, f[k + 1] = w.y, f[k + 2] = w.z, f[k + 3] = w.w;
    }
}
template <int EPV>
__device__ __forceinline__ void load_bias(const float *p, float *f)
{
#pragma unroll
    for (int k = 0; k < EPV; k += 4) {
        const f32x4_any w = *reinterpret_cast<const f32x4_any *>(p + k);
        f[k] = w.x, f[k + 1] = w.y, f[k + 2] = w.z, f[k + 3] = w.w;
    }
}

// allowed bits of the EPV entries at e (a multiple of EPV), lowest first; the entry's value or `other`
template <int EPV>
__device__ __forceinline__ uint32_t allowed_bits(const uint8_t *bits, int e)
{
    const uint32_t byte = bits[e >> 3];
    return EPV == 8 ? byte : byte >> (e & 4);
}
__device__ __forceinline__ float if_allowed(uint32_t bits, int k, float v, uint32_t other)
{
    const uint32_t on = (uint32_t)__builtin_amdgcn_sbfe((int)bits, k, 1);
    return __uint_as_float((__float_as_uint(v) & on) | (other & ~on));
}
constexpr uint32_t kMinusInfBits = 0xFF800000u;

template <typename ZT, typename UT, int NV>
__global__ __launch_bounds__(kThreads) void adjust_kernel(AdjustArgs a)
{
    constexpr int EPV = ZT::kPerVec, kWaves = kThreads / kWave;
    extern __shared__ __align__(16) float delta[];
    __shared__ float red[2 * kWaves];
    __shared__ int noted;
    uint16_t *places = reinterpret_cast<uint16_t *>(delta + a.part);
    const int64_t items = a.T * a.parts;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t t = item / a.parts, first = (item - t * a.parts) * a.part;
        const int span = (int)min((int64_t)a.part, a.V - first), full = span / EPV, rest = span - full * EPV;
        const char *row = static_cast<const char *>(a.z) + (t * a.ldz + first) * ZT::kBytes;
        char *out = a.u ? static_cast<char *>(a.u) + (t * a.ldu + first) * UT::kBytes : nullptr;
        const uint8_t *bits = a.allowed ? reinterpret_cast<const uint8_t *>(a.allowed + t * a.allowed_ld) + first / 8 : nullptr;
        const float *bias = a.bias ? a.bias + t * a.bias_ld + first : nullptr;
        uint4 raw[NV];
        uint32_t ok[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * kThreads + threadIdx.x;
            raw[i] = neg_inf_vec<ZT>();
            ok[i] = 0xFFu;
            if (v < full) {
                raw[i] = row_load<true>(row + (int64_t)v * 16);
                if (bits) ok[i] = allowed_bits<EPV>(bits, v * EPV);
            }
        }
        // (one element of what is left of the row behind the last whole vector)
        const bool last = (int)threadIdx.x < rest;
        const int le = full * EPV + threadIdx.x;
        float extra = last ? load_elem<ZT>(row, le) : -kInf;
        const RowPolicy p = row_policy(a, t);
        const bool hist = p.len > 0;
        if (hist) penalties<ZT>(a, p, row, first, span, delta, places, &noted);
        const float scale = p.inv_temperature * kLog2e;
        float f[NV][EPV], m = kLowest;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = (i * kThreads + threadIdx.x) * EPV;
            unpack<ZT>(raw[i], f[i]);
            if (e < full * EPV) {
                if (hist) {
                    float d[EPV];
                    load_lds<EPV>(delta + e, d);
#pragma unroll
                    for (int k = 0; k < EPV; ++k) f[i][k] += d[k];
                }
                if (bias) {
                    float b[EPV];
                    load_bias<EPV>(bias + e, b);
#pragma unroll
                    for (int k = 0; k < EPV; ++k) f[i][k] += b[k];
                }
            }
            if (bits && __any((~ok[i] & ((1u << EPV) - 1)) != 0))
#pragma unroll
                for (int k = 0; k < EPV; ++k) f[i][k] = if_allowed(ok[i], k, f[i][k], kMinusInfBits);
#pragma unroll
            for (int k = 0; k < EPV; ++k) m = fmaxf(m, f[i][k]);
        }
        if (last) {
            if (hist) extra += delta[le];
            if (bias) extra += bias[le];
            if (bits && !(bits[le >> 3] >> (le & 7) & 1)) extra = -kInf;
            m = fmaxf(m, extra);
        }
        if (out) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int v = i * kThreads + threadIdx.x;
                if (v < full) {
                    float u[EPV];
#pragma unroll
                    for (int k = 0; k < EPV; ++k) u[k] = f[i][k] * p.inv_temperature;
                    store_out<UT, EPV>(out + (int64_t)v * EPV * UT::kBytes, u);
                }
            }
            if (last) store_elem<UT>(out, le, extra * p.inv_temperature);
        }
        if (!a.ws_partials) continue;  // (neither log-sum-exp nor log-probs are asked for)
        // the thread that holds the chosen token leaves it for the kernel that joins the parts
        if (a.chosen) {
            const int64_t y = (int64_t)a.chosen[t] - first;
            if (y >= 0 && y < span) {
                const int vy = (int)y / EPV, ky = (int)y - vy * EPV;
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (vy < full && i * kThreads + (int)threadIdx.x == vy)
#pragma unroll
                        for (int k = 0; k < EPV; ++k)
                            if (k == ky) a.ws_chosen[t] = f[i][k];
                if (last && le == (int)y) a.ws_chosen[t] = extra;
            }
        }
        MaxSum acc = {m, exp2_hw((extra - m) * scale)};
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < EPV; ++k) acc.s += exp2_hw((f[i][k] - m) * scale);
        acc = wave_join(acc, scale);
        const int wave = threadIdx.x / kWave;
        __syncthreads();
        if ((threadIdx.x & (kWave - 1)) == 0) put(red, kWaves, wave, acc);
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kWaves; ++w) {
                MaxSum o;
                get(red, kWaves, w, o);
                acc = join(acc, o, scale);
            }
            a.ws_partials[item] = make_float2(acc.m, acc.s);
        }
    }
}

// one wavefront a row: its parts' (max, sum) to the log-sum-exp and the chosen token's log-prob
__global__ __launch_bounds__(256) void adjust_finish_kernel(AdjustArgs a)
{
    const int lane = threadIdx.x & (kWave - 1);
    for (int64_t t = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave; t < a.T; t += (int64_t)gridDim.x * 4) {
        const float inv = a.temperature ? 1.0f / a.temperature[t] : 1.0f, scale = inv * kLog2e;
        MaxSum v = {kLowest, 0.0f};
        for (int p = lane; p < a.parts; p += kWave) {
            const float2 w = a.ws_partials[t * a.parts + p];
            v = join(v, MaxSum{w.x, w.y}, scale);
        }
        v = wave_join(v, scale);
        if (lane == 0) {
            const float log_s = logf(v.s);  // (-inf where nothing is left of the row)
            if (a.lse) a.lse[t] = fmaf(v.m, inv, log_s);
            if (a.logp) {
                const int64_t y = a.chosen[t];
                float r = 0.0f;
                if (y >= 0 && y < a.V) {
                    const float u = a.ws_chosen[t];
                    r = u == -kInf ? -kInf : (u - v.m) * inv - log_s;
                }
                a.logp[t] = r;
            }
        }
    }
}

template <typename ZT, typename UT, int NV>
__global__ __launch_bounds__(kThreads) void adjust_bwd_kernel(AdjustArgs a)
{
    constexpr int EPV = ZT::kPerVec;
    extern __shared__ __align__(16) float factor[];
    const int64_t items = a.T * a.parts;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t t = item / a.parts, first = (item - t * a.parts) * a.part;
        const int span = (int)min((int64_t)a.part, a.V - first), full = span / EPV, rest = span - full * EPV;
        const char *row = static_cast<const char *>(a.z) + (t * a.ldz + first) * ZT::kBytes;
        const char *in = static_cast<const char *>(a.du) + (t * a.ldu + first) * UT::kBytes;
        char *out = static_cast<char *>(a.dz) + (t * a.lddz + first) * ZT::kBytes;
        const uint8_t *bits = a.allowed ? reinterpret_cast<const uint8_t *>(a.allowed + t * a.allowed_ld) + first / 8 : nullptr;
        float g[NV][EPV];
        uint32_t ok[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * kThreads + threadIdx.x;
            ok[i] = 0xFFu;
            if (v < full) {
                load_in<UT, EPV>(in + (int64_t)v * EPV * UT::kBytes, g[i]);
                if (bits) ok[i] = allowed_bits<EPV>(bits, v * EPV);
            }
        }
        const bool last = (int)threadIdx.x < rest;
        const int le = full * EPV + threadIdx.x;
        float extra = last ? load_elem<UT>(in, le) : 0.0f;
        const RowPolicy p = row_policy(a, t);
        const bool hist = p.len > 0 && p.repetition != 1.0f;
        if (hist) {
            const float up = p.inv_temperature * p.repetition, down = p.inv_temperature / p.repetition;
            __syncthreads();  // (the part before this one is done with the array)
            fill(factor, span, p.inv_temperature);
            __syncthreads();
            // (a token that is there twice is given the same factor twice)
            each_token(a, p, first, span, [&](int, int at) { factor[at] = load_elem<ZT>(row, at) > 0.0f ? down : up; });
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * kThreads + threadIdx.x, e = v * EPV;
            if (v < full) {
                if (hist) {
                    float d[EPV];
                    load_lds<EPV>(factor + e, d);
#pragma unroll
                    for (int k = 0; k < EPV; ++k) g[i][k] *= d[k];
                } else {
#pragma unroll
                    for (int k = 0; k < EPV; ++k) g[i][k] *= p.inv_temperature;
                }
                if (bits && __any((~ok[i] & ((1u << EPV) - 1)) != 0))
#pragma unroll
                    for (int k = 0; k < EPV; ++k) g[i][k] = if_allowed(ok[i], k, g[i][k], 0u);
                store_out<ZT, EPV>(out + (int64_t)e * ZT::kBytes, g[i]);
            }
        }
        if (last) {
            extra *= hist ? factor[le] : p.inv_temperature;
            if (bits && !(bits[le >> 3] >> (le & 7) & 1)) extra = 0.0f;
            store_elem<ZT>(out, le, extra);
        }
    }
}

template <typename ZT, typename UT, int NV>
hipError_t launch(const AdjustArgs &a, hipStream_t s)
{
    const int64_t items = a.T * a.parts, most = 1 << 20;
    const dim3 grid((unsigned)(items < most ? items : most)), block(kThreads);
    const size_t lds = a.history ? (size_t)a.part * (a.dz ? 4 : 6) : 0;
    if (a.dz) adjust_bwd_kernel<ZT, UT, NV><<<grid, block, lds, s>>>(a);
    else adjust_kernel<ZT, UT, NV><<<grid, block, lds, s>>>(a);
    return hipGetLastError();
}

template <typename ZT, typename UT>
hipError_t launch_of(const AdjustArgs &a, hipStream_t s)
{
    switch (a.vectors) {
        case 1: return launch<ZT, UT, 1>(a, s);
        case 2: return launch<ZT, UT, 2>(a, s);
        case 3: return launch<ZT, UT, 3>(a, s);
        default: return launch<ZT, UT, 4>(a, s);
    }
}

}  // namespace

hipError_t launch_adjust(AdjustArgs a, hipStream_t s)
{
    const AdjustPlan p = adjust_plan(a.T, a.V, a.z_dt == A3PO_F32 ? 4 : 2);
    a.parts = p.parts;
    a.part = p.part;
    a.vectors = p.vectors;
    hipError_t e;
    if (a.z_dt == A3PO_F32) e = a.u_dt == A3PO_F32 ? launch_of<F32, F32>(a, s) : launch_of<F32, Bf16>(a, s);
    else e = a.u_dt == A3PO_F32 ? launch_of<Bf16, F32>(a, s) : launch_of<Bf16, Bf16>(a, s);
    if (e != hipSuccess || a.dz || !a.ws_partials) return e;
    const int64_t want = (a.T + 3) / 4, most = 1 << 20;
    adjust_finish_kernel<<<dim3((unsigned)(want < most ? want : most)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace a3po
