// Logits of the policy that tokens are drawn from: penalties for repeated tokens, bias, temperature and grammar mask, with
// the log-sum-exp and the log-prob of a chosen token of the adjusted row in the same pass; and the gradient back through it.
//
//   u = z;  token in the row's history: u = u > 0 ? u / repetition : u repetition
//   u -= frequency n + presence [n > 0]      (n: how often the token is in the history behind the prompt)
//   u = (u + bias) / temperature;  not allowed: u = -inf
//   lse = log sum_j exp u_j,  logp = u_y - lse
//   dz = du / temperature * (in the history: z > 0 ? 1 / repetition : repetition), 0 where not allowed
//
// A row is cut into parts, a workgroup each: the history is counted into LDS (an integer per entry of the part: the top bit
// marks the token, the others count it behind the prompt), then the part is streamed once.  All arithmetic is fp32; what is
// stored in bfloat16 is rounded once, and lse and logp are those of the fp32 values.  The kernels are bound by memory.
#include "a3po_common.h"
#include "a3po_launch.h"

namespace a3po {
namespace {

constexpr int kThreads = kAdjustThreads;
constexpr uint32_t kSeen = 0x80000000u;
constexpr float kInf = __builtin_huge_valf();

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2), aligned(2)));

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

// The entries of [first, first + span) in the row's history: cnt[i] != 0 iff first + i is in it, its low bits count the
// occurrences behind the prompt.  Integers: the order of the additions does not matter.
__device__ __forceinline__ void count_history(const AdjustArgs &a, const RowPolicy &p, int64_t first, int span, uint32_t *cnt)
{
    __syncthreads();  // (the part before this one is done with the counts)
    for (int i = threadIdx.x; i < span; i += kThreads) cnt[i] = 0;
    __syncthreads();
    const int32_t *h = a.history + p.start;
    for (int i = threadIdx.x; i < p.len; i += kThreads) {
        const int64_t at = (int64_t)h[i] - first;
        if (at >= 0 && at < span) {
            if (i < p.prompt) atomicOr(&cnt[at], kSeen);
            else atomicAdd(&cnt[at], 1u);
        }
    }
    __syncthreads();
}

__device__ __forceinline__ float adjusted(float z, uint32_t n, float bias, const RowPolicy &p)
{
    if (n) {
        z = z > 0.0f ? z / p.repetition : z * p.repetition;
        const uint32_t out = n & ~kSeen;
        if (out) z -= fmaf(p.frequency, (float)out, p.presence);
    }
    return (z + bias) * p.inv_temperature;
}

// (max, sum) of exp; a maximum of -inf belongs to an empty sum
__device__ __forceinline__ float above(float m) { return m == -kInf ? 0.0f : m; }

__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b)
{
    MaxSum o;
    o.m = fmaxf(a.m, b.m);
    const float ref = above(o.m);
    o.s = a.s * exp2_hw((a.m - ref) * kLog2e) + b.s * exp2_hw((b.m - ref) * kLog2e);
    return o;
}

template <int N>
__device__ __forceinline__ void fold_row(MaxSum &acc, const float *f)
{
    float m = acc.m;
#pragma unroll
    for (int e = 0; e < N; ++e) m = fmaxf(m, f[e]);
    const float ref = above(m);
    float s = acc.s * exp2_hw((acc.m - ref) * kLog2e);
#pragma unroll
    for (int e = 0; e < N; ++e) s += exp2_hw((f[e] - ref) * kLog2e);
    acc.m = m;
    acc.s = s;
}

__device__ __forceinline__ MaxSum wave_join(MaxSum v)
{
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) {
        MaxSum o;
        o.m = __shfl_xor(v.m, off, kWave);
        o.s = __shfl_xor(v.s, off, kWave);
        v = join(v, o);
    }
    return v;
}

__device__ __forceinline__ float lse_of(const MaxSum &v) { return v.m == -kInf ? -kInf : v.m + logf(v.s); }
__device__ __forceinline__ float logp_of(const MaxSum &v, float u) { return u == -kInf ? -kInf : (u - v.m) - logf(v.s); }

// allowed bits of the EPV entries at e (a multiple of EPV), lowest first
template <int EPV>
__device__ __forceinline__ uint32_t allowed_bits(const uint8_t *bits, int64_t e)
{
    const uint32_t byte = bits[e >> 3];
    return EPV == 8 ? byte : byte >> (e & 4);
}
__device__ __forceinline__ bool allowed_bit(const uint8_t *bits, int64_t e) { return bits[e >> 3] >> (e & 7) & 1; }

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

template <typename ZT, typename UT, int NV>
__global__ __launch_bounds__(kThreads) void adjust_kernel(AdjustArgs a)
{
    constexpr int EPV = ZT::kPerVec, kWaves = kThreads / kWave;
    extern __shared__ __align__(16) uint32_t cnt[];
    __shared__ float red[2 * kWaves];
    const int64_t items = a.T * a.parts;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t t = item / a.parts, first = (item - t * a.parts) * a.part;
        const int span = (int)min((int64_t)a.part, a.V - first), full = span / EPV, rest = span - full * EPV;
        const char *row = static_cast<const char *>(a.z) + (t * a.ldz + first) * ZT::kBytes;
        char *out = a.u ? static_cast<char *>(a.u) + (t * a.ldu + first) * UT::kBytes : nullptr;
        uint4 raw[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * kThreads + threadIdx.x;
            raw[i] = neg_inf_vec<ZT>();
            if (v < full) raw[i] = row_load<true>(row + (int64_t)v * 16);
        }
        const bool last = (int)threadIdx.x < rest;
        const int le = full * EPV + threadIdx.x;
        const float z_extra = last ? load_elem<ZT>(row, le) : -kInf;
        const RowPolicy p = row_policy(a, t);
        const bool hist = p.len > 0;
        if (hist) count_history(a, p, first, span, cnt);
        const float *bias = a.bias ? a.bias + t * a.bias_ld + first : nullptr;
        const uint8_t *bits = a.allowed ? reinterpret_cast<const uint8_t *>(a.allowed + t * a.allowed_ld) + first / 8 : nullptr;
        MaxSum acc = {-kInf, 0.0f};
        // the part that holds the chosen token looks it up again at the end
        const int64_t y = a.chosen ? (int64_t)a.chosen[t] - first : -1;
        float u_y = -kInf;
        bool has_y = false;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * kThreads + threadIdx.x, e = v * EPV;
            if (v < full) {
                float f[EPV];
                unpack<ZT>(raw[i], f);
                uint32_t n[EPV];
#pragma unroll
                for (int k = 0; k < EPV; ++k) n[k] = hist ? cnt[e + k] : 0u;
                float b[EPV];
#pragma unroll
                for (int k = 0; k < EPV; ++k) b[k] = 0.0f;
                if (bias)
#pragma unroll
                    for (int k = 0; k < EPV; k += 4) {
                        const f32x4_any w = *reinterpret_cast<const f32x4_any *>(bias + e + k);
                        b[k] = w.x, b[k + 1] = w.y, b[k + 2] = w.z, b[k + 3] = w.w;
                    }
                const uint32_t ok = bits ? allowed_bits<EPV>(bits, e) : ~0u;
#pragma unroll
                for (int k = 0; k < EPV; ++k) {
                    f[k] = adjusted(f[k], n[k], b[k], p);
                    if (!(ok >> k & 1)) f[k] = -kInf;
                    if (e + k == y) u_y = f[k], has_y = true;
                }
                if (out) store_out<UT, EPV>(out + (int64_t)e * UT::kBytes, f);
                fold_row<EPV>(acc, f);
            }
        }
        if (last) {
            float f = adjusted(z_extra, hist ? cnt[le] : 0u, bias ? bias[le] : 0.0f, p);
            if (bits && !allowed_bit(bits, le)) f = -kInf;
            if (le == y) u_y = f, has_y = true;
            if (out) store_elem<UT>(out, le, f);
            fold_row<1>(acc, &f);
        }
        if (has_y) a.ws_chosen[t] = u_y;
        if (!a.ws_partials) continue;  // (neither log-sum-exp nor log-probs are asked for)
        acc = wave_join(acc);
        const int wave = threadIdx.x / kWave;
        __syncthreads();
        if ((threadIdx.x & (kWave - 1)) == 0) put(red, kWaves, wave, acc);
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kWaves; ++w) {
                MaxSum o;
                get(red, kWaves, w, o);
                acc = join(acc, o);
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
        MaxSum v = {-kInf, 0.0f};
        for (int p = lane; p < a.parts; p += kWave) {
            const float2 w = a.ws_partials[t * a.parts + p];
            v = join(v, MaxSum{w.x, w.y});
        }
        v = wave_join(v);
        if (lane == 0) {
            if (a.lse) a.lse[t] = lse_of(v);
            if (a.logp) {
                const int64_t y = a.chosen[t];
                a.logp[t] = y >= 0 && y < a.V ? logp_of(v, a.ws_chosen[t]) : 0.0f;
            }
        }
    }
}

template <typename ZT, typename UT, int NV>
__global__ __launch_bounds__(kThreads) void adjust_bwd_kernel(AdjustArgs a)
{
    constexpr int EPV = ZT::kPerVec;
    extern __shared__ __align__(16) uint32_t cnt[];
    const int64_t items = a.T * a.parts;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t t = item / a.parts, first = (item - t * a.parts) * a.part;
        const int span = (int)min((int64_t)a.part, a.V - first), full = span / EPV, rest = span - full * EPV;
        const char *row = static_cast<const char *>(a.z) + (t * a.ldz + first) * ZT::kBytes;
        const char *in = static_cast<const char *>(a.du) + (t * a.ldu + first) * UT::kBytes;
        char *out = static_cast<char *>(a.dz) + (t * a.lddz + first) * ZT::kBytes;
        float g[NV][EPV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * kThreads + threadIdx.x;
            if (v < full) load_in<UT, EPV>(in + (int64_t)v * EPV * UT::kBytes, g[i]);
        }
        const bool last = (int)threadIdx.x < rest;
        const int le = full * EPV + threadIdx.x;
        const float g_extra = last ? load_elem<UT>(in, le) : 0.0f;
        const RowPolicy p = row_policy(a, t);
        const bool hist = p.len > 0 && p.repetition != 1.0f;
        if (hist) count_history(a, p, first, span, cnt);
        const uint8_t *bits = a.allowed ? reinterpret_cast<const uint8_t *>(a.allowed + t * a.allowed_ld) + first / 8 : nullptr;
        const float up = p.repetition, down = 1.0f / p.repetition;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * kThreads + threadIdx.x, e = v * EPV;
            if (v < full) {
                uint32_t n[EPV], any = 0;
#pragma unroll
                for (int k = 0; k < EPV; ++k) {
                    n[k] = hist ? cnt[e + k] : 0u;
                    any |= n[k];
                }
#pragma unroll
                for (int k = 0; k < EPV; ++k) g[i][k] *= p.inv_temperature;
                if (any) {  // the logit's sign is asked for here alone
                    float z[EPV];
                    unpack<ZT>(row_load<true, true>(row + (int64_t)v * 16), z);
#pragma unroll
                    for (int k = 0; k < EPV; ++k)
                        if (n[k]) g[i][k] *= z[k] > 0.0f ? down : up;
                }
                const uint32_t ok = bits ? allowed_bits<EPV>(bits, e) : ~0u;
#pragma unroll
                for (int k = 0; k < EPV; ++k)
                    if (!(ok >> k & 1)) g[i][k] = 0.0f;
                store_out<ZT, EPV>(out + (int64_t)e * ZT::kBytes, g[i]);
            }
        }
        if (last) {
            float f = g_extra * p.inv_temperature;
            if (hist && cnt[le]) f *= load_elem<ZT>(row, le) > 0.0f ? down : up;
            if (bits && !allowed_bit(bits, le)) f = 0.0f;
            store_elem<ZT>(out, le, f);
        }
    }
}

template <typename ZT, typename UT, int NV>
hipError_t launch(const AdjustArgs &a, hipStream_t s)
{
    const int64_t items = a.T * a.parts, most = 1 << 20;
    const dim3 grid((unsigned)(items < most ? items : most)), block(kThreads);
    const size_t lds = a.history ? (size_t)a.part * 4 : 0;
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
