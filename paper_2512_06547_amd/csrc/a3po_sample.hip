// Tokens drawn from the policy: every row's logits are cut by top-k, top-p and min-p, and the entry in whose part of the kept
// mass the drawn number falls is the token.
//
//   x = (z - max z) / temperature,  w = e^x
//   order: larger logits first, the lower index first among equal ones.  Each cut keeps a beginning of that order, so that all of
//   them together are one border (key, ties): kept are the entries above the key and the first `ties` of those at it.
//   token = first v with sum_{kept j <= v} w_j > uniform * sum_kept w
//
// Sums of weights are whole numbers: a weight is rounded to a multiple of 2^-shift of the largest's, shift = 62 - log2 V (50 at
// most), so that V of them fit 64 bits, additions commute, atomics on them included, and the sum of the kept that the border was
// found with is the sum that the number is drawn in.
#include "a3po_common.h"
#include "a3po_launch.h"

namespace a3po {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr int kBins = 4096;
constexpr uint32_t kKeyOfNegInf = 0x007FFFFFu, kAll = 0xFFFFFFFFu;

// e^x: 2^(i / 32) from a table (one entry a pair of LDS banks: lanes never wait for one another), the rest of the exponent by a
// series whose first term left out, (ln 2 / 64)^6 / 720, is 2^-48
struct Weigh {
    double max, unit;     // unit: 32 log2(e) / temperature
    const double *table;  // 2^(shift + i / 32)
    __device__ __forceinline__ double operator()(float z) const
    {
        constexpr double a1 = 0.69314718055994530942 / 32, a2 = a1 * a1 / 2, a3 = a2 * a1 / 3, a4 = a3 * a1 / 4, a5 = a4 * a1 / 5;
        constexpr double kRound = 6755399441055744.0;  // 1.5 * 2^52: the sum's low word is the whole number
        const double y = fmax(((double)z - max) * unit, -32000.0);
        const double t = y + kRound;
        const int n = __double2loint(t);
        const double r = y - (t - kRound);
        const double b = table[n & 31];
        const double scale = __hiloint2double(__double2hiint(b) + ((n >> 5) << 20), __double2loint(b));
        const double q = r * (a1 + r * (a2 + r * (a3 + r * (a4 + r * a5))));
        return scale + scale * q;
    }
    __device__ __forceinline__ uint64_t whole(float z) const
    {
        return (uint64_t)__double_as_longlong((*this)(z) + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
    }
};

// orders floats as whole numbers; -0 and 0 are one
__device__ __forceinline__ uint32_t key_of(float z)
{
    const uint32_t u = __float_as_uint(z + 0.0f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

template <typename T>
__device__ __forceinline__ T wave_scan(T v)  // inclusive
{
    const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const T up = __shfl_up(v, off, kWave);
        if (lane >= off) v += up;
    }
    return v;
}

struct Shared {
    uint64_t mass[kBins];
    uint32_t count[kBins];
    uint64_t block_mass[kSampleBlocks];
    uint32_t block_count[kSampleBlocks];
    double table[32];
    uint64_t wave_mass[kWaves];
    uint32_t wave_count[kWaves];
    uint64_t found_mass;
    uint32_t found_digit, found_count;
};

// inclusive over the workgroup, with the totals; LDS of the waves' sums is free again behind the next barrier
__device__ __forceinline__ void block_scan(Shared &sh, uint64_t &mass, uint32_t &count, uint64_t &mass_total, uint32_t &count_total)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    mass = wave_scan((unsigned long long)mass);
    count = wave_scan(count);
    __syncthreads();
    if (lane == kWave - 1) sh.wave_mass[wave] = mass, sh.wave_count[wave] = count;
    __syncthreads();
    uint64_t m = 0;
    uint32_t c = 0;
    mass_total = 0, count_total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) m += sh.wave_mass[w], c += sh.wave_count[w];
        mass_total += sh.wave_mass[w], count_total += sh.wave_count[w];
    }
    mass += m, count += c;
}

template <typename DT>
struct Row {
    static constexpr int kEpv = DT::kPerVec;
    const char *p;
    int64_t V;
    int steps, blocks;  // of 64 vectors a block; blocks

    __device__ __forceinline__ int64_t first(int b, int s) const
    {
        return ((int64_t)b * steps + s) * (kWave * kEpv) + (int)(threadIdx.x & (kWave - 1)) * kEpv;
    }
    __device__ __forceinline__ void load(int64_t e, float *f) const  // -inf behind the row's end
    {
        if (e + kEpv <= V) {
            unpack<DT>(row_load<true, true>(p + e * DT::kBytes), f);
        } else {
#pragma unroll
            for (int k = 0; k < kEpv; ++k) f[k] = e + k < V ? load_elem<DT>(p, e + k) : -__builtin_huge_valf();
        }
    }
    // f(values, first entry, block) of every 64 vectors of the row, a wavefront each
    template <typename F>
    __device__ __forceinline__ void each(F f) const
    {
        for (int b = threadIdx.x / kWave; b < blocks; b += kWaves)
            for (int s = 0; s < steps; ++s) {
                float v[kEpv];
                const int64_t e = first(b, s);
                load(e, v);
                f(v, e, b);
            }
    }
};

struct Border {
    uint32_t key, ties;  // kAll: every entry at the key
};
__device__ __forceinline__ Border tighter(Border a, Border b)
{
    if (a.key != b.key) return a.key > b.key ? a : b;
    return Border{a.key, min(a.ties, b.ties)};
}

template <typename DT>
struct Picker {
    Shared &sh;
    Row<DT> row;
    Weigh weigh;

    // counts and masses of the entries whose key's bits above shift + bits are `prefix`, by their next `bits`
    __device__ void histogram(uint32_t prefix, int shift, int bits)
    {
        __syncthreads();
        for (int i = threadIdx.x; i < kBins; i += kThreads) sh.mass[i] = 0, sh.count[i] = 0;
        __syncthreads();
        const uint32_t mask = (1u << bits) - 1;
        row.each([&](const float *v, int64_t, int) {
#pragma unroll
            for (int k = 0; k < Row<DT>::kEpv; ++k) {
                const uint32_t key = key_of(v[k]);
                if (key > kKeyOfNegInf && (bits + shift == 32 || key >> (shift + bits) == prefix)) {
                    const uint32_t d = key >> shift & mask;
                    atomicAdd(&sh.count[d], 1u);
                    atomicAdd(reinterpret_cast<unsigned long long *>(&sh.mass[d]), (unsigned long long)weigh.whole(v[k]));
                }
            }
        });
        __syncthreads();
    }
    // the bin, from the top, in which the running count (or mass) reaches `target`; adds what is above it to `count`, `mass`
    template <bool MASS>
    __device__ uint32_t find(uint64_t target, uint64_t &mass, uint32_t &count, uint64_t &mass_total, uint32_t &count_total)
    {
        constexpr int kEach = kBins / kThreads;
        uint64_t m[kEach], ms = 0;
        uint32_t c[kEach], cs = 0;
        const int top = kBins - 1 - (int)threadIdx.x * kEach;
#pragma unroll
        for (int i = 0; i < kEach; ++i) m[i] = sh.mass[top - i], c[i] = sh.count[top - i], ms += m[i], cs += c[i];
        uint64_t mi = ms;
        uint32_t ci = cs;
        block_scan(sh, mi, ci, mass_total, count_total);
        uint64_t ma = mass + mi - ms;
        uint32_t ca = count + ci - cs;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const bool before = MASS ? ma < target : ca < target;
            if (before && (MASS ? ma + m[i] >= target : (uint64_t)ca + c[i] >= target))
                sh.found_digit = top - i, sh.found_mass = ma, sh.found_count = ca;
            ma += m[i], ca += c[i];
        }
        __syncthreads();
        mass = sh.found_mass, count = sh.found_count;
        return sh.found_digit;
    }
    // the border that leaves the first `target` entries (or the fewest whose mass is `target`), the first level's bins being
    // there; mass: that of what it leaves
    template <bool MASS>
    __device__ Border select(uint64_t target, uint64_t &mass)
    {
        uint64_t above = 0, mt;
        uint32_t count = 0, ct;
        uint32_t prefix = find<MASS>(target, above, count, mt, ct);
        histogram(prefix, 8, 12);
        uint32_t digit = find<MASS>(target, above, count, mt, ct);
        prefix = prefix << 12 | digit;
        if constexpr (DT::kBytes == 4) {
            histogram(prefix, 0, 8);
            digit = find<MASS>(target, above, count, mt, ct);
            prefix = prefix << 8 | digit;
        } else {
            prefix = prefix << 8 | (prefix >> 23 ? 0u : 0xFFu);  // (bfloat16's low bits are zeros, inverted where it is negative)
        }
        const uint32_t equal = sh.count[digit];
        const uint64_t each = sh.mass[digit] / equal;  // (equal logits have equal weights)
        uint64_t ties = MASS ? (target - above + each - 1) / (each ? each : 1) : target - count;
        if (ties > equal) ties = equal;
        mass = above + ties * each;
        return Border{prefix, ties == equal ? kAll : (uint32_t)ties};
    }
};

// bit k: entry k is kept; `seen`: entries at the border before this wavefront's 64 vectors, counted on where that matters
template <int EPV>
__device__ __forceinline__ uint32_t kept_of(const float *v, Border border, uint32_t &seen)
{
    uint32_t above = 0, at = 0;
#pragma unroll
    for (int k = 0; k < EPV; ++k) {
        const uint32_t key = key_of(v[k]);
        above |= (key > border.key ? 1u : 0u) << k;
        at |= (key == border.key ? 1u : 0u) << k;
    }
    if (border.ties == kAll) return above | at;
    if (border.ties == 0 || !__any(at)) return above;
    const uint32_t own = __popc(at), upto = wave_scan(own);
    uint32_t rank = seen + upto - own;
#pragma unroll
    for (int k = 0; k < EPV; ++k)
        if (at >> k & 1) above |= (rank++ < border.ties ? 1u : 0u) << k;
    seen += __shfl(upto, kWave - 1, kWave);
    return above;
}

// One workgroup a row, all of its passes from memory.
template <typename DT>
__global__ __launch_bounds__(kThreads) void sample_rows_kernel(SampleArgs a)
{
    __shared__ Shared sh;
    constexpr int EPV = DT::kPerVec;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    if (tid < 32) sh.table[tid] = ldexp(exp2((double)tid / 32), a.shift);
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        Row<DT> row{reinterpret_cast<const char *>(a.z) + t * a.ld * DT::kBytes, a.V, a.steps, a.blocks};
        // ---- the maximum
        float top = -__builtin_huge_valf();
        bool bad = false;
        row.each([&](const float *v, int64_t, int) {
#pragma unroll
            for (int k = 0; k < EPV; ++k) top = fmaxf(top, v[k]), bad |= !(v[k] < __builtin_huge_valf());
        });
#pragma unroll
        for (int off = kWave / 2; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
        bad = __any(bad);
        __syncthreads();  // (the row before this one is done with everything)
        if (lane == 0) sh.wave_count[wave] = __float_as_uint(bad ? __builtin_nanf("") : top);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float o = __uint_as_float(sh.wave_count[w]);
            bad |= o != o;
            top = fmaxf(top, o);
        }
        __syncthreads();
        // ---- the row's policy
        float tau = a.temperature ? a.temperature[t] : 1.0f;
        int64_t k = a.top_k ? a.top_k[t] : 0;
        const float p = a.top_p ? a.top_p[t] : 1.0f, min_p = a.min_p ? a.min_p[t] : 0.0f;
        float u = a.uniform[t];
        bad |= !(tau >= 0.0f) || p != p || min_p != min_p || u != u;
        if (tau == 0.0f) tau = 1.0f, k = 1;
        if (bad || top == -__builtin_huge_valf()) {
            if (a.allowed)
                for (int64_t w = tid; w < (a.V + 31) / 32; w += kThreads) a.allowed[t * a.allowed_ld + w] = 0;
            if (tid == 0) {
                const float none = bad ? __builtin_nanf("") : -__builtin_huge_valf();
                a.token[t] = -1;
                if (a.logp) a.logp[t] = none;
                if (a.logp_full) a.logp_full[t] = none;
                if (a.kept) a.kept[t] = 0;
            }
            continue;
        }
        const Weigh weigh{(double)top, 46.166241308446828384 / (double)tau, sh.table};  // 32 log2(e)
        Picker<DT> pick{sh, row, weigh};
        // ---- the border
        Border border{kKeyOfNegInf, 0};
        const bool by_k = k > 0 && k < a.V, by_p = p < 1.0f;
        if (by_k || by_p) {
            pick.histogram(0, 20, 12);
            uint64_t mass = 0, total;
            uint32_t count = 0, finite;
            pick.template find<true>(1, mass, count, total, finite);
            if (by_k && k < finite) {
                border = pick.template select<false>((uint64_t)k, total);
                if (by_p) pick.histogram(0, 20, 12);
            }
            if (by_p) {
                const double need = ceil((double)fmaxf(p, 0.0f) * (double)total);
                uint64_t target = need < 1.0 ? 1 : (uint64_t)need;
                if (target > total) target = total;
                border = tighter(border, pick.template select<true>(target, mass));
            }
        }
        if (min_p > 0.0f) {
            // the smallest float at or above max + temperature ln(min_p)
            const double least = (double)top + (double)tau * log((double)fminf(min_p, 1.0f));
            float zt = (float)least;
            if ((double)zt < least) zt = nextafterf(zt, __builtin_huge_valf());
            if (zt > -__builtin_huge_valf()) border = tighter(border, Border{key_of(zt), kAll});
        }
        const bool partial = border.ties != kAll && border.ties != 0;
        // ---- entries at the border before each block, where not all are kept
        uint64_t mass = 0, total;
        uint32_t count = 0, kept;
        __syncthreads();
        if (tid < kSampleBlocks) sh.block_count[tid] = 0, sh.block_mass[tid] = 0;
        __syncthreads();
        if (partial) {
            row.each([&](const float *v, int64_t, int b) {
                int n = 0;
#pragma unroll
                for (int e = 0; e < EPV; ++e) n += __popcll(__ballot(key_of(v[e]) == border.key));
                if (lane == 0 && n) sh.block_count[b] += n;
            });
            __syncthreads();
            const uint32_t own = sh.block_count[tid];
            count = own;
            block_scan(sh, mass, count, total, kept);
            sh.block_count[tid] = count - own;
            __syncthreads();
        }
        // ---- mass and number of the kept in each block, their bits
        uint64_t full = 0;
        uint32_t mine = 0;
        for (int b = wave; b < row.blocks; b += kWaves) {
            uint32_t seen = sh.block_count[b];
            uint64_t in_block = 0;
            for (int s = 0; s < row.steps; ++s) {
                float v[EPV];
                const int64_t e = row.first(b, s);
                row.load(e, v);
                const uint32_t bits = kept_of<EPV>(v, border, seen);
#pragma unroll
                for (int i = 0; i < EPV; ++i) {
                    const uint64_t w = weigh.whole(v[i]);
                    full += w;
                    if (bits >> i & 1) in_block += w;
                }
                mine += __popc(bits);
                if (a.allowed) {
                    uint32_t word = bits << (e & 31);
#pragma unroll
                    for (int off = 1; off < 32 / EPV; off <<= 1) word |= __shfl_xor(word, off, kWave);
                    if ((e & 31) == 0 && e < a.V) a.allowed[t * a.allowed_ld + (e >> 5)] = (int32_t)word;
                }
            }
            const uint64_t sum = wave_scan((unsigned long long)in_block);
            if (lane == kWave - 1) sh.block_mass[b] = sum;
        }
        uint64_t all = full;
        uint64_t full_total;
        block_scan(sh, all, mine, full_total, kept);
        __syncthreads();
        const uint64_t own = sh.block_mass[tid];
        mass = own, count = 0;
        uint32_t none;
        block_scan(sh, mass, count, total, none);
        // ---- the block, then the entry, in whose part of the sum the number falls
        u = fminf(fmaxf(u, 0.0f), 1.0f - 5.9604645e-8f);
        const uint64_t target = (uint64_t)((double)u * (double)total);
        if (mass > target && mass - own <= target) sh.found_digit = tid, sh.found_mass = target - (mass - own);
        __syncthreads();
        if (wave == 0) {
            const int b = (int)sh.found_digit;
            uint64_t left = sh.found_mass;
            uint32_t seen = sh.block_count[b];
            for (int s = 0; s < row.steps; ++s) {
                float v[EPV];
                const int64_t e = row.first(b, s);
                row.load(e, v);
                const uint32_t bits = kept_of<EPV>(v, border, seen);
                uint64_t sum = 0;
#pragma unroll
                for (int i = 0; i < EPV; ++i) sum += bits >> i & 1 ? weigh.whole(v[i]) : 0;
                const uint64_t upto = wave_scan((unsigned long long)sum);
                const uint64_t here = __ballot(upto > left);
                if (here) {
                    if (lane == __builtin_ctzll(here)) {
                        uint64_t at = upto - sum;
                        int i = 0;
                        for (; i < EPV - 1; ++i) {
                            at += bits >> i & 1 ? weigh.whole(v[i]) : 0;
                            if (at > left) break;
                        }
                        float z = v[0];
#pragma unroll
                        for (int j = 1; j < EPV; ++j) z = j == i ? v[j] : z;
                        const double x = ((double)z - (double)top) / (double)tau, unit = a.shift * 0.69314718055994530942;
                        a.token[t] = (int32_t)(e + i);
                        if (a.logp) a.logp[t] = (float)(x - (log((double)total) - unit));
                        if (a.logp_full) a.logp_full[t] = (float)(x - (log((double)full_total) - unit));
                        if (a.kept) a.kept[t] = (int32_t)kept;
                    }
                    break;
                }
                left -= __shfl((unsigned long long)upto, kWave - 1, kWave);
            }
        }
    }
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, hipStream_t s)
{
    const int grid = (int)(a.T < (1 << 20) ? a.T : 1 << 20);
    if (a.dt == A3PO_F32) sample_rows_kernel<F32><<<grid, kThreads, 0, s>>>(a);
    else sample_rows_kernel<Bf16><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace a3po
