// Logits of the policy that tokens are drawn from: penalties for repeated tokens, bias, temperature and grammar mask, with
// the log-sum-exp and the log-prob of a chosen token of the adjusted row in the same pass; and the gradient back through it.
//
//   u = z;  token in the row's history: u = u > 0 ? u / repetition : u repetition
//   u -= frequency n + presence [n > 0]      (n: how often the token is in the history behind the prompt)
//   u = (u + bias) / temperature;  not allowed: u = -inf
//   lse = log sum_j exp u_j,  logp = u_y - lse
//   dz = du / temperature * (in the history: z > 0 ? 1 / repetition : repetition), 0 where not allowed
//
// A workgroup takes a row, or a part of one where rows are few.  The row's history becomes a bit per entry in LDS.  Forward,
// entries without the bit are folded from registers as they stream by, and the others, few, are taken one a thread
// afterwards: the bits number them, the part's tokens, noted while they were marked, are counted by those numbers (integers: no
// order of additions), and the entries join the sum and the output.  A test per entry with the penalties behind it costs more
// than the exponential, and the work on the history, the reductions and the row's parameters cost what some forty entries a
// thread do, so that rows are not cut further than it takes to fill the chip (scoring of 8,192 x 50,001 bfloat16: a test per
// entry, four parts a row 1,055 us; a penalty per entry in LDS 553; bits, four parts 735; bits, whole rows 306; now 227).
// What bounds it: scoring, 819 MB in 228 us (3.6 TB/s), the vector instructions, active in 91 % of a compute unit's cycles, 17 an entry
// with the history's (with workgroups of 512, 280 us: 212 without a history, 31 for the bits, 16 for the counts, 36 for the
// entries; 4,096 x 151,936 without one 237 us, 5.3 TB/s); decoding, 64 x 151,936 to fp32 with 16,384 tokens of history, 34 us, the passes over
// the history (18 us without one); written rows, 4,096 x 151,936 bfloat16 to fp32, memory where there is no history (805 us, 4.6 TB/s),
// and the work on one of up to 2,047 tokens, in series with its row, 235 us more; the gradient, two streams and little else, memory:
// 8,192 x 151,936 4.98 GB in 1,050 us (4.7 TB/s, what a large copy reaches).
// Rows are read and written through the caches: the entries of the history are fetched a second time (non-temporal: 301 for
// 281 us, decoding 42 for 38), and the next kernel reads what is written here.
// Maximum and sum of exp are taken before the temperature, which then is part of the exponent's scale.  All arithmetic is
// fp32; what is stored in bfloat16 is rounded once, and lse and logp are those of the fp32 values.
#include "a3po_common.h"
#include "a3po_launch.h"

namespace a3po {
namespace {

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

// A part of a row: every 2^shift-th block of 512 entries from the `index`-th on.  (Runs of entries would leave most of a
// history, which holds the vocabulary's first tokens by far the most often, to the first part.)  Parts number their entries
// by themselves; `id` is an entry's place in the row.
struct Part {
    static constexpr int kBlock = 512;
    int shift, index;
    int span;  // entries
    __device__ __forceinline__ Part(const AdjustArgs &a, int part) : shift(a.parts_shift), index(part)
    {
        const int64_t blocks = (a.V + kBlock - 1) / kBlock, mine = (blocks - part + (1 << shift) - 1) >> shift;
        const bool holds_last = ((blocks - 1) & ((1 << shift) - 1)) == part;
        span = mine > 0 ? (int)(mine * kBlock - (holds_last ? blocks * kBlock - a.V : 0)) : 0;
    }
    __device__ __forceinline__ uint32_t id(int at) const { return ((((uint32_t)at >> 9) << shift | index) << 9) | (at & (kBlock - 1)); }
    // the entry of token `token`, if it is one of the part's (V: the row's length)
    __device__ __forceinline__ bool has(int32_t token, int64_t V, uint32_t &at) const
    {
        const uint32_t t = (uint32_t)token, block = t >> 9;
        at = (block >> shift) << 9 | (t & (kBlock - 1));
        return t < (uint32_t)V && (block & ((1u << shift) - 1)) == (uint32_t)index;
    }
};

// f(places, valid, output) for the tokens of the row's history, four at a time: places[k] is the k-th one's entry in the part
// if bit k of `valid` says that it is one of the part's; bit k of `output`: it is behind the prompt
template <int THREADS, typename F>
__device__ __forceinline__ void each_tokens(const AdjustArgs &a, const RowPolicy &p, const Part &part, F f)
{
    const int32_t *h = a.history + p.start;
    constexpr uint32_t kLoads = 4, kRound = THREADS * 4 * kLoads;
    const uint32_t len = (uint32_t)p.len, prompt = (uint32_t)max(p.prompt, 0), lane = threadIdx.x;
    auto one = [&](int32_t id, uint32_t at_history, int k, uint32_t(&at)[4], uint32_t &valid, uint32_t &output) {
        valid |= (part.has(id, a.V, at[k]) ? 1u : 0u) << k;
        output |= (at_history >= prompt ? 1u : 0u) << k;
    };
    uint32_t i = 0;  // (unsigned: lengths end below 2^31, the places tried beyond them below 2^32)
    for (; len - i >= kRound; i += kRound) {
        i32x4_any v[kLoads];
#pragma unroll
        for (uint32_t j = 0; j < kLoads; ++j) v[j] = *reinterpret_cast<const i32x4_any *>(h + i + (j * THREADS + lane) * 4);
#pragma unroll
        for (uint32_t j = 0; j < kLoads; ++j) {
            uint32_t at[4], valid = 0, output = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) one(v[j][k], i + (j * THREADS + lane) * 4 + k, k, at, valid, output);
            f(at, valid, output);
        }
    }
    for (; i < len; i += THREADS * kLoads) {
        int32_t v[kLoads];
#pragma unroll
        for (uint32_t j = 0; j < kLoads; ++j) {
            const uint32_t at = i + j * THREADS + lane;
            v[j] = at < len ? h[at] : -1;
        }
        uint32_t at[4], valid = 0, output = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) one(v[k], i + k * THREADS + lane, k, at, valid, output);
        f(at, valid, output);
    }
}

// The part's entries that are in the row's history: a bit each, and the numbers of those entries.
template <int THREADS>
struct Seen {
    static constexpr int kBlock = 16;  // words whose numbers share a base
    uint32_t *words;                   // [part / 32]
    uint32_t *bases;                   // [part / 512]
    uint16_t *before;                  // [part / 32], within the block
    int nwords;

    __device__ __forceinline__ Seen(char *lds, int part)
        : words(reinterpret_cast<uint32_t *>(lds)), bases(words + part / 32),
          before(reinterpret_cast<uint16_t *>(bases + part / 512)), nwords(part / 32)
    {
    }

    // With a `list` of `room` tokens for the wavefront, its tokens that are the part's are noted there, the output's with the
    // top bit; returns how many they are, those behind the list's end included.
    template <bool LIST>
    __device__ __forceinline__ int mark(const AdjustArgs &a, const RowPolicy &p, const Part &part, uint32_t *list, int room)
    {
        int listed = 0;
        __syncthreads();  // (the part before this one is done with the bits)
        for (int w = threadIdx.x; w < nwords / 4; w += THREADS) reinterpret_cast<uint4 *>(words)[w] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        each_tokens<THREADS>(a, p, part, [&](const uint32_t(&at)[4], uint32_t valid, uint32_t output) {
            // (most of a text's tokens are there already: looking first spares the atomics that all would aim at a few words)
            uint32_t have[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) have[k] = valid >> k & 1 ? words[at[k] >> 5] : ~0u;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (!(have[k] >> (at[k] & 31) & 1)) atomicOr(&words[at[k] >> 5], 1u << (at[k] & 31));
            if constexpr (LIST)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint64_t mine = __ballot(valid >> k & 1);
                    const int to = listed + __builtin_amdgcn_mbcnt_hi((uint32_t)(mine >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mine, 0));
                    if ((valid >> k & 1) && to < room) list[to] = at[k] | (output >> k) << 31;
                    listed += __popcll(mine);
                }
        });
        __syncthreads();
        return listed;
    }
    // numbers the marked entries in ascending order; returns how many there are (numbers are there behind the next barrier)
    __device__ __forceinline__ int count(int *waves)
    {
        const int tid = threadIdx.x, wave = tid / kWave, lane = tid & (kWave - 1);
        int own = 0;
        if (tid < nwords / kBlock)  // (a part has at most a block a thread)
#pragma unroll
            for (int k = 0; k < kBlock; k += 4) {
                const uint4 w = reinterpret_cast<const uint4 *>(words)[(tid * kBlock + k) / 4];
                uint16_t *to = before + tid * kBlock + k;
                to[0] = (uint16_t)own, own += __popc(w.x);
                to[1] = (uint16_t)own, own += __popc(w.y);
                to[2] = (uint16_t)own, own += __popc(w.z);
                to[3] = (uint16_t)own, own += __popc(w.w);
            }
        int sum = own;
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const int up = __shfl_up(sum, off, kWave);
            if (lane >= off) sum += up;
        }
        if (lane == kWave - 1) waves[wave] = sum;
        __syncthreads();
        int base = 0, total = 0;
#pragma unroll
        for (int w = 0; w < THREADS / kWave; ++w) {
            base += w < wave ? waves[w] : 0;
            total += waves[w];
        }
        if (tid < nwords / kBlock) bases[tid] = (uint32_t)(base + sum - own);
        return total;
    }
    template <int EPV>
    __device__ __forceinline__ uint32_t bits(int e) const  // of the EPV entries at e, a multiple of EPV
    {
        const uint32_t byte = reinterpret_cast<const uint8_t *>(words)[e >> 3];
        return EPV == 8 ? byte : byte >> (e & 4) & 15u;
    }
    __device__ __forceinline__ bool bit(int e) const { return words[e >> 5] >> (e & 31) & 1; }
    __device__ __forceinline__ int number_of_word(int w) const { return (int)bases[w / kBlock] + before[w]; }
    __device__ __forceinline__ int number(uint32_t at) const
    {
        return number_of_word((int)(at >> 5)) + __popc(words[at >> 5] & ((1u << (at & 31)) - 1));
    }
};

// (max, sum) pairs: sum_j exp((v_j - max) / temperature); nothing yet is (lowest, 0)
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float scale)
{
    MaxSum o;
    o.m = fmaxf(a.m, b.m);
    o.s = a.s * exp2_hw((a.m - o.m) * scale) + b.s * exp2_hw((b.m - o.m) * scale);
    return o;
}
template <int LANES = kWave>
__device__ __forceinline__ MaxSum wave_join(MaxSum v, float scale)
{
    float m = v.m;
#pragma unroll
    for (int off = LANES / 2; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, kWave));
    float s = v.s * exp2_hw((v.m - m) * scale);
#pragma unroll
    for (int off = LANES / 2; off > 0; off >>= 1) s += __shfl_xor(s, off, kWave);
    return MaxSum{m, s};
}

template <typename UT, int EPV>
__device__ __forceinline__ void store_out(char *p, const float *f)
{
    if constexpr (UT::kBytes * EPV >= 16) {
#pragma unroll
        for (int k = 0; k < EPV; k += UT::kPerVec) {
            const uint4 v = pack<UT>(f + k);
            const u32x4_t t = {v.x, v.y, v.z, v.w};
            *reinterpret_cast<u32x4_elem_t *>(p + k * UT::kBytes) = t;
        }
    } else {
        const u32x2_t t = {pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])};
        *reinterpret_cast<u32x2_t *>(p) = t;
    }
}

// EPV elements of type UT as they are in memory, and widened
template <typename UT, int EPV>
struct Raw {
    static constexpr int kWords = UT::kBytes * EPV / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const char *p)
    {
        if constexpr (kWords >= 4) {
#pragma unroll
            for (int k = 0; k < kWords; k += 4) {
                const uint4 v = row_load<true, true>(p + 4 * k);
                w[k] = v.x, w[k + 1] = v.y, w[k + 2] = v.z, w[k + 3] = v.w;
            }
        } else {
            const u32x2_t t = *reinterpret_cast<const u32x2_t *>(p);
            w[0] = t.x, w[1] = t.y;
        }
    }
    __device__ __forceinline__ void widen(float *f) const
    {
#pragma unroll
        for (int k = 0; k < kWords; ++k) {
            if constexpr (UT::kBytes == 4) f[k] = __uint_as_float(w[k]);
            else f[2 * k] = __uint_as_float(w[k] << 16), f[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
        }
    }
};

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
// (two instructions; from a comparison or a mask in C the compiler makes three)
__device__ __forceinline__ float if_allowed(uint32_t bits, int k, float v, float other)
{
    const int on = __builtin_amdgcn_sbfe((int)bits, k, 1);
    float r;
    asm("v_bfi_b32 %0, %1, %2, %3" : "=v"(r) : "v"(on), "v"(v), "v"(other));
    return r;
}
// the largest of three (fmaxf makes a quiet NaN of each operand first, an instruction each; a NaN shows in the sums)
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// Folds a thread's values into its (max, sum), m being the new maximum.  exp2(f s - c) is one instruction less than
// exp2((f - m) s) and, with c = m s rounded, differs from it by the factor 2^(m s - c) alone, which the sum is freed of
// at once: the exponent is rounded relative to f - m as before.  From |m s| = 2^23 on, where that factor could leave the range
// (values masked by large numbers, all but greedy temperatures, infinities), the difference comes first.
template <int N>
__device__ __forceinline__ void fold_values(MaxSum &acc, const float (&f)[N], float m, float scale)
{
    const float c = m * scale;
    float s = 0.0f;
    if (__any(!(fabsf(c) < 8388608.0f))) {
#pragma unroll
        for (int k = 0; k < N; ++k) s += exp2_hw((f[k] - m) * scale);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) s += exp2_hw(fmaf(f[k], scale, -c));
        s *= exp2_hw(-fmaf(m, scale, -c));
    }
    acc.s = fmaf(acc.s, exp2_hw((acc.m - m) * scale), s);
    acc.m = m;
}

// what is told of a row: of its (max, sum), and of the chosen token's adjusted logit before the temperature
__device__ __forceinline__ void finish_row(const AdjustArgs &a, int64_t t, MaxSum v, float inv_temperature, float u)
{
    const float log_s = logf(v.s);  // (-inf where nothing is left of the row)
    if (a.lse) a.lse[t] = fmaf(v.m, inv_temperature, log_s);
    if (a.logp) {
        const int64_t y = a.chosen[t];
        // (a row of which nothing is left has -inf - -inf; a sum that is NaN stays one whatever the token's logit)
        const bool never = u == -kInf && v.s >= 0.0f;
        a.logp[t] = y < 0 || y >= a.V ? 0.0f : never ? -kInf : (u - v.m) * inv_temperature - log_s;
    }
}

template <typename ZT, typename UT, int NV, int THREADS>
__global__ __launch_bounds__(THREADS, 4) void adjust_kernel(AdjustArgs a)
{
    constexpr int EPV = ZT::kPerVec, kWaves = THREADS / kWave, kStep = THREADS * EPV * NV;
    constexpr uint32_t kAll = (1u << EPV) - 1;
    extern __shared__ __align__(16) char lds[];
    __shared__ float red[2 * kWaves];
    __shared__ int waves[kWaves];
    __shared__ float u_chosen;
    Seen<THREADS> seen(lds, a.part);
    const int room = adjust_numbers(a.part);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane_e = (threadIdx.x & (kWave - 1)) * EPV;
    uint32_t *counts = reinterpret_cast<uint32_t *>(lds + adjust_seen_bytes(a.part, true)), *places = counts + room;
    const int list_room = adjust_listed(a.part, THREADS);
    uint32_t *list = places + room + wave * list_room;
    const int64_t items = a.T << a.parts_shift;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t t = item >> a.parts_shift;
        const Part part(a, (int)(item & ((1 << a.parts_shift) - 1)));
        const int whole = part.span / EPV * EPV, rest = part.span - whole;
        const char *row = static_cast<const char *>(a.z) + t * a.ldz * ZT::kBytes;
        char *out = a.u ? static_cast<char *>(a.u) + t * a.ldu * UT::kBytes : nullptr;
        const uint8_t *bits = a.allowed ? reinterpret_cast<const uint8_t *>(a.allowed + t * a.allowed_ld) : nullptr;
        const float *bias = a.bias ? a.bias + t * a.bias_ld : nullptr;
        Raw<ZT, EPV> next[NV];
        uint32_t next_ok[NV];
        // (a wavefront's vectors lie in one block: its place in the row is one number)
        auto first_of = [&](int at, int i) { return at + (i * kWaves + wave) * (kWave * EPV); };
        auto fetch = [&](int at) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int e = first_of(at, i);
                if (e + lane_e < whole) {
                    const uint32_t id = part.id(e);
                    next[i].load(row + (uint64_t)id * ZT::kBytes + lane_e * ZT::kBytes);
                    if (bits) next_ok[i] = allowed_bits<EPV>(bits + id / 8, lane_e) & kAll;
                }
            }
        };
        fetch(0);
        // (one element of what is left of the row behind the last whole vector)
        const bool last = (int)threadIdx.x < rest;
        const int le = whole + threadIdx.x;
        const uint32_t id_last = part.id(le);
        const float z_last = last ? load_elem<ZT>(row, id_last) : -kInf;
        const RowPolicy p = row_policy(a, t);
        uint32_t y_at = 0;
        const int y = a.logp && part.has(a.chosen[t], a.V, y_at) ? (int)y_at : -1;
        const float scale = p.inv_temperature * kLog2e;
        const bool hist = p.len > 0 && (p.repetition != 1.0f || p.frequency != 0.0f || p.presence != 0.0f);
        const int listed = hist ? __builtin_amdgcn_readfirstlane(seen.template mark<true>(a, p, part, list, list_room)) : 0;

        MaxSum acc = {kLowest, 0.0f};
        for (int at = 0; at < whole; at += kStep) {
            Raw<ZT, EPV> raw[NV];
            uint32_t ok[NV];
#pragma unroll
            for (int i = 0; i < NV; ++i) raw[i] = next[i], ok[i] = next_ok[i];
            if (at + kStep < whole) fetch(at + kStep);
            float f[NV * EPV], m = acc.m;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int first = first_of(at, i), e = first + lane_e;
                const uint32_t id = part.id(first);
                if (e >= whole) {
#pragma unroll
                    for (int k = 0; k < EPV; ++k) f[i * EPV + k] = -kInf;
                    continue;
                }
                raw[i].widen(f + i * EPV);
                const uint32_t later = hist ? seen.template bits<EPV>(e) : 0u;
                if (bias) {
                    float b[EPV];
                    load_bias<EPV>(bias + id + lane_e, b);
#pragma unroll
                    for (int k = 0; k < EPV; ++k) f[i * EPV + k] += b[k];
                }
                if (bits && __any(ok[i] != kAll))
#pragma unroll
                    for (int k = 0; k < EPV; ++k) f[i * EPV + k] = if_allowed(ok[i], k, f[i * EPV + k], -kInf);
                if (out) {
                    float u[EPV];
#pragma unroll
                    for (int k = 0; k < EPV; ++k) u[k] = f[i * EPV + k] * p.inv_temperature;
                    if (later) {  // (their logits stay there for now: out may be the logits' own place)
                        float z[EPV];
                        raw[i].widen(z);
#pragma unroll
                        for (int k = 0; k < EPV; ++k) u[k] = later >> k & 1 ? z[k] : u[k];
                    }
                    store_out<UT, EPV>(out + (uint64_t)id * UT::kBytes + lane_e * UT::kBytes, u);
                }
                if (y >= e && y < e + EPV)
#pragma unroll
                    for (int k = 0; k < EPV; ++k)
                        if (e + k == y && !(later >> k & 1)) u_chosen = f[i * EPV + k];
                if (__any(later != 0))
#pragma unroll
                    for (int k = 0; k < EPV; ++k) f[i * EPV + k] = if_allowed(~later, k, f[i * EPV + k], -kInf);
#pragma unroll
                for (int k = 0; k < EPV; k += 2) m = max3(m, f[i * EPV + k], f[i * EPV + k + 1]);
            }
            fold_values(acc, f, m, scale);
        }
        auto bias_of = [&](uint32_t id) { return bias ? bias[id] : 0.0f; };
        auto ok_of = [&](uint32_t id) { return !bits || (bits[id >> 3] >> (id & 7) & 1); };
        auto put_out = [&](int at, float v) {
            if (out) store_elem<UT>(out, part.id(at), v * p.inv_temperature);
            if (at == y) u_chosen = v;
        };
        // (infinity and NaN make the sum NaN)
        auto one_of = [](float v) { return v == -kInf ? 0.0f : v - v + 1.0f; };
        if (last) {
            if (!(hist && seen.bit(le))) {
                const float v = ok_of(id_last) ? z_last + bias_of(id_last) : -kInf;
                put_out(le, v);
                acc = join(acc, MaxSum{fmaxf(v, kLowest), one_of(v)}, scale);
            } else if (out) {
                store_elem<UT>(out, id_last, z_last);
            }
        }
        // the entries of the history, one a thread
        const int numbers = hist ? seen.count(waves) : 0;
        const float down = 1.0f / p.repetition;
        for (int base = 0; base < numbers; base += room) {
            const int many = min(numbers - base, room);
            __syncthreads();  // (the numbers are there, the row is written, the counts before these are done with)
            for (int i = threadIdx.x; i < many; i += THREADS) counts[i] = 0;
            __syncthreads();
            // (a token that is there more than once notes the same place)
            auto count_tokens = [&](const uint32_t(&at)[4], uint32_t valid, uint32_t output) {
                int n[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) n[k] = valid >> k & 1 ? seen.number(at[k]) - base : -1;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (n[k] >= 0 && n[k] < room) {
                        places[n[k]] = at[k];
                        if (output >> k & 1) atomicAdd(&counts[n[k]], 1u);
                    }
            };
            if (listed <= list_room) {
                for (int i = threadIdx.x & (kWave - 1); i < listed; i += 4 * kWave) {
                    uint32_t at[4], valid = 0, output = 0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int from = i + k * kWave;
                        const uint32_t v = list[min(from, listed - 1)];
                        at[k] = v & 0x7FFFFFFFu;
                        valid |= (from < listed ? 1u : 0u) << k;
                        output |= v >> 31 << k;
                    }
                    count_tokens(at, valid, output);
                }
            } else {
                each_tokens<THREADS>(a, p, part, count_tokens);
            }
            __syncthreads();
            constexpr int kBatch = 4;  // (a thread's loads in flight)
            for (int i = threadIdx.x; i < many; i += THREADS * kBatch) {
                int at[kBatch];
                float v[kBatch], b[kBatch], m = acc.m;
                bool ok[kBatch];
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    at[k] = (int)places[min(i + k * THREADS, many - 1)];
                    const uint32_t id = part.id(at[k]);
                    v[k] = load_elem<ZT>(row, id);
                    b[k] = bias_of(id);
                    ok[k] = ok_of(id);
                }
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    const bool there = i + k * THREADS < many;
                    const uint32_t n = there ? counts[i + k * THREADS] : 0;
                    v[k] *= v[k] > 0.0f ? down : p.repetition;
                    if (n) v[k] -= fmaf(p.frequency, (float)n, p.presence);
                    v[k] = there && ok[k] ? v[k] + b[k] : -kInf;
                    if (there) put_out(at[k], v[k]);
                    m = fmaxf(m, v[k]);
                }
                fold_values(acc, v, m, scale);
            }
        }
        if (!a.ws_partials) continue;  // (neither log-sum-exp nor log-probs are asked for)
        acc = wave_join(acc, scale);
        __syncthreads();
        if ((threadIdx.x & (kWave - 1)) == 0) put(red, kWaves, wave, acc);
        __syncthreads();
        if (threadIdx.x < kWaves) {
            get(red, kWaves, threadIdx.x, acc);
            acc = wave_join<kWaves>(acc, scale);
            if (threadIdx.x == 0) {
                if (a.parts_shift == 0) {
                    finish_row(a, t, acc, p.inv_temperature, u_chosen);
                } else {
                    a.ws_partials[item] = make_float2(acc.m, acc.s);
                    if (y >= 0) a.ws_chosen[t] = u_chosen;
                }
            }
        }
        if (item + gridDim.x < items) __syncthreads();  // (u_chosen is read)
    }
}

// one wavefront a row: its parts' (max, sum) to the log-sum-exp and the chosen token's log-prob
__global__ __launch_bounds__(256) void adjust_finish_kernel(AdjustArgs a)
{
    const int lane = threadIdx.x & (kWave - 1);
    for (int64_t t = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave; t < a.T; t += (int64_t)gridDim.x * 4) {
        const float inv = a.temperature ? 1.0f / a.temperature[t] : 1.0f, scale = inv * kLog2e;
        MaxSum v = {kLowest, 0.0f};
        for (int p = lane; p < 1 << a.parts_shift; p += kWave) {
            const float2 w = a.ws_partials[(t << a.parts_shift) + p];
            v = join(v, MaxSum{w.x, w.y}, scale);
        }
        v = wave_join(v, scale);
        if (lane == 0) finish_row(a, t, v, inv, a.ws_chosen[t]);
    }
}

template <typename ZT, typename UT, int NV>
__global__ __launch_bounds__(kAdjustThreads) void adjust_bwd_kernel(AdjustArgs a)
{
    constexpr int EPV = ZT::kPerVec, kWaves = kAdjustThreads / kWave, kStep = kAdjustThreads * EPV * NV;
    constexpr uint32_t kAll = (1u << EPV) - 1;
    extern __shared__ __align__(16) char lds[];
    Seen<kAdjustThreads> seen(lds, a.part);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane_e = (threadIdx.x & (kWave - 1)) * EPV;
    const int64_t items = a.T << a.parts_shift;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t t = item >> a.parts_shift;
        const Part part(a, (int)(item & ((1 << a.parts_shift) - 1)));
        const int whole = part.span / EPV * EPV, rest = part.span - whole;
        const char *row = static_cast<const char *>(a.z) + t * a.ldz * ZT::kBytes;
        const char *in = static_cast<const char *>(a.du) + t * a.ldu * UT::kBytes;
        char *out = static_cast<char *>(a.dz) + t * a.lddz * ZT::kBytes;
        const uint8_t *bits = a.allowed ? reinterpret_cast<const uint8_t *>(a.allowed + t * a.allowed_ld) : nullptr;
        Raw<UT, EPV> next[NV];
        uint32_t next_ok[NV];
        auto first_of = [&](int at, int i) { return at + (i * kWaves + wave) * (kWave * EPV); };
        auto fetch = [&](int at) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int e = first_of(at, i);
                if (e + lane_e < whole) {
                    const uint32_t id = part.id(e);
                    next[i].load(in + (uint64_t)id * UT::kBytes + lane_e * UT::kBytes);
                    if (bits) next_ok[i] = allowed_bits<EPV>(bits + id / 8, lane_e) & kAll;
                }
            }
        };
        fetch(0);
        const bool last = (int)threadIdx.x < rest;
        const int le = whole + threadIdx.x;
        const uint32_t id_last = part.id(le);
        const float g_last = last ? load_elem<UT>(in, id_last) : 0.0f;
        const RowPolicy p = row_policy(a, t);
        const bool hist = p.len > 0 && p.repetition != 1.0f;
        if (hist) seen.mark<false>(a, p, part, nullptr, 0);
        const float up = p.inv_temperature * p.repetition, down = p.inv_temperature / p.repetition;
        for (int at = 0; at < whole; at += kStep) {
            Raw<UT, EPV> raw[NV];
            uint32_t ok[NV], hit[NV];
            uint4 z[NV];
            // logits of vectors that hold an entry of the history: asked for together, before the next gradients
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int first = first_of(at, i), e = first + lane_e;
                raw[i] = next[i], ok[i] = next_ok[i];
                hit[i] = hist && e < whole ? seen.bits<EPV>(e) : 0u;
                if (hit[i]) z[i] = row_load<true, true>(row + (uint64_t)part.id(first) * ZT::kBytes + lane_e * ZT::kBytes);
            }
            if (at + kStep < whole) fetch(at + kStep);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int first = first_of(at, i);
                if (first + lane_e >= whole) continue;
                float g[EPV];
                raw[i].widen(g);
                if (hit[i]) {
                    float w[EPV];
                    unpack<ZT>(z[i], w);
#pragma unroll
                    for (int k = 0; k < EPV; ++k) g[k] *= hit[i] >> k & 1 ? (w[k] > 0.0f ? down : up) : p.inv_temperature;
                } else {
#pragma unroll
                    for (int k = 0; k < EPV; ++k) g[k] *= p.inv_temperature;
                }
                if (bits && __any(ok[i] != kAll))
#pragma unroll
                    for (int k = 0; k < EPV; ++k) g[k] = if_allowed(ok[i], k, g[k], 0.0f);
                store_out<ZT, EPV>(out + (uint64_t)part.id(first) * ZT::kBytes + lane_e * ZT::kBytes, g);
            }
        }
        if (last) {
            float f = g_last * p.inv_temperature;
            if (hist && seen.bit(le)) f = g_last * (load_elem<ZT>(row, id_last) > 0.0f ? down : up);
            if (bits && !(bits[id_last >> 3] >> (id_last & 7) & 1)) f = 0.0f;
            store_elem<ZT>(out, id_last, f);
        }
    }
}

template <typename ZT, typename UT>
hipError_t launch(const AdjustArgs &a, int threads, hipStream_t s)
{
    const int64_t items = a.T << a.parts_shift, most = 1 << 20;
    const dim3 grid((unsigned)(items < most ? items : most)), block(threads);
    const size_t lds = a.history ? adjust_lds(a.part, threads, a.dz) : 0;
    if (a.dz) adjust_bwd_kernel<ZT, UT, 2><<<grid, block, lds, s>>>(a);
    else if (threads == kAdjustThreads) adjust_kernel<ZT, UT, 2, kAdjustThreads><<<grid, block, lds, s>>>(a);
    else adjust_kernel<ZT, UT, 2, kAdjustThreads / 2><<<grid, block, lds, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_adjust(AdjustArgs a, hipStream_t s)
{
    const AdjustPlan p = adjust_plan(a.T, a.V, a.z_dt == A3PO_F32 ? 4 : 2, a.dz != nullptr);
    const int threads = a.dz ? kAdjustThreads : adjust_threads(a.T, p, a.u != nullptr);
    a.parts_shift = p.shift;
    a.part = p.part;
    hipError_t e;
    if (a.z_dt == A3PO_F32) e = a.u_dt == A3PO_F32 ? launch<F32, F32>(a, threads, s) : launch<F32, Bf16>(a, threads, s);
    else e = a.u_dt == A3PO_F32 ? launch<Bf16, F32>(a, threads, s) : launch<Bf16, Bf16>(a, threads, s);
    if (e != hipSuccess || a.dz || !a.ws_partials || a.parts_shift == 0) return e;
    const int64_t want = (a.T + 3) / 4, most = 1 << 20;
    adjust_finish_kernel<<<dim3((unsigned)(want < most ? want : most)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace a3po
