// Tokens drawn from the policy: every row's logits are cut by top-k, top-p and min-p, and the entry in whose part of the kept
// mass the drawn number falls is the token.
//
//   x = (z - max z) / temperature,  w = e^x
//   order: larger logits first, the lower index first among equal ones.  Each cut keeps a beginning of that order, so that all of
//   them together are one border, the last entry kept: its logit and its index.
//   token = first v with sum_{kept j <= v} w_j > uniform * sum_kept w
//
// A row is cut into parts of 8,192 entries, a workgroup each.
//   parts:   the part's maximum and the sum of its weights; where the row is cut, counts and sums of its entries in bins of 1/16
//            power of two of their weight, on one grid for all parts, so that parts add up
//   rows:    uncut, the token: the part, then the entry, in whose part of the sum the drawn number falls.  Cut, the bin that the
//            border is in
//   gather:  the entries down to that bin, where they are few, else that bin's alone: parts without any are not read again
//   finish:  the border among those entries, and the token
// Rows that this does not settle (borders among very many equal logits, or 2^-32 below the largest weight) are gone over by one
// workgroup as often as their cuts ask.
//
// In a bin, weights are relative to the bin's and added as whole numbers of 2^-36, their count above them in the same 64 bits: one
// atomic an entry.  Everywhere else that entries are counted by atomics weights are multiples of 2^-shift of the row's largest,
// shift = 62 - log2 V (50 at most), so that V of them fit 64 bits.  Both make additions commute.
#include "a3po_common.h"
#include "a3po_launch.h"

namespace a3po {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr int kBins = 4096;
constexpr uint32_t kKeyOfNegInf = 0x007FFFFFu;
constexpr int kPartThreads = 256, kPartWaves = kPartThreads / kWave;

constexpr float kInf = __builtin_huge_valf();

// 2^(i / 32)
__device__ const double kTable[32] = {
    0x1.0000000000000p+0, 0x1.059b0d3158574p+0, 0x1.0b5586cf9890fp+0, 0x1.11301d0125b51p+0,
    0x1.172b83c7d517bp+0, 0x1.1d4873168b9aap+0, 0x1.2387a6e756238p+0, 0x1.29e9df51fdee1p+0,
    0x1.306fe0a31b715p+0, 0x1.371a7373aa9cbp+0, 0x1.3dea64c123422p+0, 0x1.44e086061892dp+0,
    0x1.4bfdad5362a27p+0, 0x1.5342b569d4f82p+0, 0x1.5ab07dd485429p+0, 0x1.6247eb03a5585p+0,
    0x1.6a09e667f3bcdp+0, 0x1.71f75e8ec5f74p+0, 0x1.7a11473eb0187p+0, 0x1.82589994cce13p+0,
    0x1.8ace5422aa0dbp+0, 0x1.93737b0cdc5e5p+0, 0x1.9c49182a3f090p+0, 0x1.a5503b23e255dp+0,
    0x1.ae89f995ad3adp+0, 0x1.b7f76f2fb5e47p+0, 0x1.c199bdd85529cp+0, 0x1.cb720dcef9069p+0,
    0x1.d5818dcfba487p+0, 0x1.dfc97337b9b5fp+0, 0x1.ea4afa2a490dap+0, 0x1.f50765b6e4540p+0};

// a b + c, the constant c from scalar registers (left to itself the compiler copies it to the sum's registers every time)
__device__ __forceinline__ double fma_const(double a, double b, double c)
{
    double d;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "s"(c));
    return d;
}

// e^x: 2^(i / 32) from a table (one entry a pair of LDS banks: lanes never wait for one another), the rest of the exponent by a
// series whose first term left out, (ln 2 / 64)^6 / 720, is 2^-48
struct Weigh {
    double max, unit;     // unit: 32 log2(e) / temperature
    const double *table;  // 2^(i / 32) times what the result is to be scaled by
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
        double q = r * a5 + a4;
        q = fma_const(q, r, a3), q = fma_const(q, r, a2), q = fma_const(q, r, a1);
        return fma(scale, r * q, scale);
    }
    __device__ __forceinline__ uint64_t whole(float z) const
    {
        return (uint64_t)__double_as_longlong((*this)(z) + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
    }
};
constexpr double kUnit = 46.166241308446828384;  // 32 log2(e)

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
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, kWave));
    return v;
}
template <typename T>
__device__ __forceinline__ T wave_sum(T v)
{
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
    return v;
}

// the last entry of the order that is kept
struct Border {
    uint32_t key;
    int32_t last;
    __device__ __forceinline__ bool keeps(float z, int32_t e) const
    {
        const uint32_t k = key_of(z);
        return k > key || (k == key && e <= last);
    }
};
constexpr int32_t kAnyIndex = 0x7FFFFFFF;
__device__ __forceinline__ Border tighter(Border a, Border b)
{
    if (a.key != b.key) return a.key > b.key ? a : b;
    return Border{a.key, min(a.last, b.last)};
}

// What the row's arrays say, absent ones being neutral.
struct Policy {
    float tau, p, min_p, u;
    int64_t k;
    bool bad, by_k, by_p, by_min;
    __device__ __forceinline__ Policy(const SampleArgs &a, int64_t t)
        : tau(a.temperature ? a.temperature[t] : 1.0f), p(a.top_p ? a.top_p[t] : 1.0f), min_p(a.min_p ? a.min_p[t] : 0.0f),
          u(a.uniform[t]), k(a.top_k ? a.top_k[t] : 0)
    {
        bad = !(tau >= 0.0f) || p != p || min_p != min_p || u != u;
        if (tau == 0.0f) tau = 1.0f, k = 1;
        by_k = k > 0 && k < a.V;
        by_p = p < 1.0f;
        by_min = min_p > 0.0f;
    }
    __device__ __forceinline__ bool cut() const { return by_k || by_p || by_min; }
};

// ---- parts -------------------------------------------------------------------------------------------------------------

// A part's entries in registers: a wavefront's are together, its v-th vectors behind its v - 1st; -inf behind the row's end.
template <typename DT>
struct PartEntries {
    static constexpr int EPV = DT::kPerVec, kVectors = kSamplePart / (kPartThreads * EPV), kEach = kVectors * EPV;
    uint4 raw[kVectors];  // (as they are in memory: bfloat16 takes half the registers)
    __device__ __forceinline__ static int first() { return (int)(threadIdx.x / kWave) * (kSamplePart / kPartWaves) + (int)(threadIdx.x & (kWave - 1)) * EPV; }
    __device__ __forceinline__ void load(const char *z, int left)
    {
#pragma unroll
        for (int v = 0; v < kVectors; ++v) {
            const int e = first() + v * kWave * EPV;
            if (e + EPV <= left) {
                raw[v] = row_load<true, true>(z + e * DT::kBytes);
            } else {
                float f[EPV];
#pragma unroll
                for (int k = 0; k < EPV; ++k) f[k] = e + k < left ? load_elem<DT>(z, e + k) : -kInf;
                raw[v] = pack<DT>(f);
            }
        }
    }
    // f(value, its number among the lane's) of every entry
    template <typename F>
    __device__ __forceinline__ void each(F f) const
    {
#pragma unroll
        for (int v = 0; v < kVectors; ++v) {
            float x[EPV];
            uint4 r = raw[v];
            asm volatile("" : "+v"(r.x), "+v"(r.y), "+v"(r.z), "+v"(r.w));  // (nothing of one pass is kept for the next)
            unpack<DT>(r, x);
#pragma unroll
            for (int k = 0; k < EPV; ++k) f(x[k], v * EPV + k);
            __builtin_amdgcn_sched_barrier(0);  // (all vectors at once take more registers than they save time)
        }
    }
};

// Places on the grid: the whole number next to z times 16 log2(e) / temperature, in 64 bits so that larger logits never have
// smaller places; what is further below zero than kFar counts as there.
constexpr double kGrid = kUnit / 2, kFar = -1.5e9, kNear = 1.0e9, kRound = 6755399441055744.0;
__device__ __forceinline__ int place_of(float z, double grid) { return __double2loint(fmax((double)z * grid, kFar) + kRound); }
// in a bin's sum: the count in the upper 14 bits, weights times 2^36 below (8,192 of them, each below 1.03, are below 2^50; the bin's middle is 1)
constexpr int kWeightBits = 50;
constexpr uint64_t kWeightMask = (1ull << kWeightBits) - 1;

template <typename DT>
__global__ __launch_bounds__(kPartThreads, 4) void sample_parts_kernel(SampleArgs a, int64_t row0, int64_t rows)
{
    using Entries = PartEntries<DT>;
    __shared__ double table[32];
    __shared__ uint64_t bins[kSampleBins];
    __shared__ float wave_top[kPartWaves];
    __shared__ double wave_mass[kPartWaves];
    __shared__ uint32_t wave_count[kPartWaves], wave_last[kPartWaves];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    if (tid < 32) table[tid] = kTable[tid];
    for (int64_t i = blockIdx.x; i < rows * a.parts; i += gridDim.x) {
        const int64_t r = i / a.parts, t = row0 + r;
        const int64_t begin = (i - r * a.parts) * kSamplePart;
        Entries z;
        z.load(reinterpret_cast<const char *>(a.z) + (t * a.ld + begin) * DT::kBytes, (int)min(a.V - begin, (int64_t)kSamplePart));
        const Policy policy(a, t);
        float top = -kInf;
        bool bad = false;
        z.each([&](float x, int) { top = fmaxf(top, x), bad |= !(x < kInf); });
        top = wave_max(top);
        if (__any(bad)) top = __builtin_nanf("");
        __syncthreads();  // (the part before this one is done with the shared arrays)
        if (lane == 0) wave_top[wave] = top;
#pragma unroll
        for (int b = tid; b < kSampleBins; b += kPartThreads) bins[b] = 0;
        __syncthreads();
        top = wave_top[0], bad = top != top;
#pragma unroll
        for (int w = 1; w < kPartWaves; ++w) bad |= wave_top[w] != wave_top[w], top = fmaxf(top, wave_top[w]);
        SamplePart out = {};
        out.max = bad ? __builtin_nanf("") : top;
        if (bad || policy.bad || top == -kInf) {  // (nothing to sum)
            if (tid == 0) a.part[i] = out;
            continue;
        }
        double mass = 0.0;
        uint32_t count = 0;
        if (!policy.cut()) {
            const Weigh weigh{(double)top, kUnit / (double)policy.tau, table};
            z.each([&](float x, int) {
                mass += weigh(x);  // (-inf: 2^-1000)
                asm volatile("" : "+v"(mass));  // (here, not where it is used)
            });
            if (a.kept) z.each([&](float x, int) { count += x > -kInf ? 1u : 0u; });
        } else {
            const double grid = kGrid / (double)policy.tau;
            const bool near = fabs((double)top * grid) < kNear;  // (beyond it the row is gone over)
            const int place = near ? place_of(top, grid) : 0;
            out.place = near ? place : kSampleFar;
            float tail = 0.0f;
            if (near) {
                uint32_t furthest = 0;
                z.each([&](float x, int) {
                    constexpr double a1 = 0.69314718055994530942 / 16, a2 = a1 * a1 / 2, a3 = a2 * a1 / 3, a4 = a3 * a1 / 4, a5 = a4 * a1 / 5;
                    constexpr double kOne = 68719476736.0, kWhole = 4503599627370496.0;  // 2^36, 2^52
                    const double y = fmax((double)x * grid, kFar), n = y + kRound, q = y - (n - kRound);
                    const uint32_t bin = (uint32_t)(place - __double2loint(n));
                    double w = q * (a5 * kOne) + a4 * kOne;
                    w = fma_const(w, q, a3 * kOne), w = fma_const(w, q, a2 * kOne), w = fma_const(w, q, a1 * kOne), w = fma_const(w, q, kOne + kWhole);
                    furthest = max(furthest, bin);
                    if (bin < kSampleBins) {
                        const uint64_t add = (uint64_t)(((uint32_t)__double2hiint(w) & 0xFFFFFu) | 1u << (kWeightBits - 32)) << 32 | (uint32_t)__double2loint(w);
                        atomicAdd(reinterpret_cast<unsigned long long *>(&bins[bin]), (unsigned long long)add);
                    }
                });
                // what lies behind the bins is below 2^-32 of the largest, all of it below 2^-19: what fp32 loses of that is below 2^-38
                if (__any(furthest >= kSampleBins))
                    z.each([&](float x, int) {
                        const double y = fmax((double)x * grid, kFar), n = y + kRound, q = y - (n - kRound);
                        const uint32_t bin = (uint32_t)(place - __double2loint(n));
                        const bool behind = bin >= kSampleBins && x > -kInf;
                        tail += behind ? exp2_hw(((float)q - (float)bin) * 0.0625f) : 0.0f;
                        count += behind ? 1u : 0u;
                        asm volatile("" : "+v"(tail), "+v"(count));
                    });
            }
            mass = (double)tail;
        }
        mass = wave_sum(mass);
        __syncthreads();  // (the bins are whole)
        uint32_t last = 0;
        if (out.place != kSampleFar)
#pragma unroll
            for (int b = tid; b < kSampleBins; b += kPartThreads) {
                const uint64_t sum = bins[b];
                if (sum) last = b + 1, count += (uint32_t)(sum >> kWeightBits);
            }
        count = wave_sum(count);
#pragma unroll
        for (int off = kWave / 2; off > 0; off >>= 1) last = max(last, (uint32_t)__shfl_xor((int)last, off, kWave));
        if (lane == 0) wave_mass[wave] = mass, wave_count[wave] = count, wave_last[wave] = last;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kPartWaves; ++w) out.mass += wave_mass[w], out.count += wave_count[w], out.bins = max(out.bins, wave_last[w]);
        for (int b = tid; b < (int)out.bins; b += kPartThreads) a.bins[i * kSampleBins + b] = bins[b];
        if (tid == 0) a.part[i] = out;
    }
}

// ---- gather ------------------------------------------------------------------------------------------------------------

template <typename DT>
__global__ __launch_bounds__(kPartThreads, 4) void sample_gather_kernel(SampleArgs a, int64_t row0, int64_t rows)
{
    using Entries = PartEntries<DT>;
    constexpr int EPV = Entries::EPV, kVectors = Entries::kVectors;
    __shared__ uint32_t wave_count[kPartWaves], start;
    __shared__ double wave_mass[kPartWaves];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    for (int64_t i = blockIdx.x; i < rows * a.parts; i += gridDim.x) {
        const int64_t r = i / a.parts, t = row0 + r;
        SampleRow &row = a.row[r];
        if (row.mode != kSampleFew && row.mode != kSampleBin) continue;
        SampleSegment out = {};
        const SamplePart part = a.part[i];
        // the part's own bins that are looked for: up to `last`, of many only that one
        const int shift = part.max > -kInf ? row.place - part.place : 0;  // part's bin 0 is the row's bin `shift`
        const bool few = row.mode == kSampleFew, all = row.bin == kSampleAll;
        const int last = all ? kSampleAll : row.bin - shift;
        if (part.max > -kInf && last >= 0) {
            uint32_t n = 0;
            double above = 0.0;
            for (int b = tid; b < (int)part.bins; b += kPartThreads) {
                const uint64_t v = a.bins[i * kSampleBins + b];
                if (few ? b <= last : b == last) n += (uint32_t)(v >> kWeightBits);
                if (!few && b < last) above += (double)(v & kWeightMask) * exp2(-0.0625 * (b + shift));
            }
            if (all) n = tid == 0 ? part.count : 0;
            n = wave_sum(n);
            above = wave_sum(above);
            __syncthreads();
            if (lane == 0) wave_count[wave] = n, wave_mass[wave] = above;
            __syncthreads();
            n = 0;
#pragma unroll
            for (int w = 0; w < kPartWaves; ++w) n += wave_count[w], out.above += wave_mass[w];
            out.listed = n;
            if (n > 0) {
                Policy policy(a, t);
                const double grid = kGrid / (double)policy.tau;
                const int64_t begin = (i - r * a.parts) * kSamplePart;
                Entries z;
                z.load(reinterpret_cast<const char *>(a.z) + (t * a.ld + begin) * DT::kBytes, (int)min(a.V - begin, (int64_t)kSamplePart));
                const int lowest = all ? -0x7FFFFFFF : row.place - row.bin, highest = few ? 0x7FFFFFFF : lowest;
                uint32_t taken = 0;  // a bit an entry
                z.each([&](float x, int k) {
                    const int p = place_of(x, grid);
                    taken |= (x > -kInf && p >= lowest && p <= highest ? 1u : 0u) << k;
                });
                // how many of each 64 vectors are before a lane's, 16 bits each
                uint32_t pos[(kVectors + 1) / 2], sum[(kVectors + 1) / 2], in_wave = 0;
#pragma unroll
                for (int w = 0; w < (kVectors + 1) / 2; ++w) {
                    uint32_t own = 0;
#pragma unroll
                    for (int h = 0; h < 2; ++h) own |= (uint32_t)__popc(taken >> ((2 * w + h) * EPV) & ((1u << EPV) - 1)) << (16 * h);
                    const uint32_t scan = wave_scan(own);
                    pos[w] = scan - own;
                    sum[w] = __shfl(scan, kWave - 1, kWave);
                    in_wave += (sum[w] & 0xFFFFu) + (sum[w] >> 16);
                }
                __syncthreads();  // (wave_count has been read)
                if (lane == 0) wave_count[wave] = in_wave;
                if (tid == 0) start = atomicAdd(&row.cursor, n);
                __syncthreads();
                out.start = start;
                uint32_t base = start;
#pragma unroll
                for (int w = 0; w < kPartWaves; ++w) base += w < wave ? wave_count[w] : 0;
                uint2 *list = a.list + r * kSampleListed;
#pragma unroll
                for (int v = 0; v < kVectors; ++v) {
                    uint32_t to = base + (pos[v / 2] >> (16 * (v & 1)) & 0xFFFFu);
                    float x[EPV];
                    unpack<DT>(z.raw[v], x);
#pragma unroll
                    for (int k = 0; k < EPV; ++k)
                        if (taken >> (v * EPV + k) & 1u) {
                            if (to < kSampleListed)
                                list[to] = make_uint2(__float_as_uint(x[k]), (uint32_t)(begin + Entries::first() + v * kWave * EPV + k));
                            ++to;
                        }
                    base += sum[v / 2] >> (16 * (v & 1)) & 0xFFFFu;
                }
            }
        }
        if (tid == 0) a.segment[i] = out;
    }
}

// ---- rows and finish -------------------------------------------------------------------------------------------------

struct Scans {
    double table[32];
    uint64_t wave_mass[kWaves];
    double wave_sum[kWaves];
    uint32_t wave_count[kWaves];
    float wave_top[kWaves];
    uint64_t found_mass;
    uint32_t found_digit, found_count, gathered;
    Border found;
};
struct Shared : Scans {
    union {
        struct {  // entries of the row by bits of their keys
            uint64_t mass[kBins];
            uint32_t count[kBins];
        } key;
        struct {
            float value[kSampleListed];
            int32_t index[kSampleListed];
            uint64_t bin_mass[kThreads];
            uint32_t bin_count[kThreads];
        } list;
    };
    uint64_t block_mass[kSampleBlocks];
    uint32_t block_count[kSampleBlocks];
};

// inclusive over the workgroup, with the totals
__device__ __forceinline__ void block_scan(Scans &sh, uint64_t &mass, uint32_t &count, uint64_t &mass_total, uint32_t &count_total)
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
#pragma unroll 4
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) m += sh.wave_mass[w], c += sh.wave_count[w];
        mass_total += sh.wave_mass[w], count_total += sh.wave_count[w];
    }
    mass += m, count += c;
}
__device__ __forceinline__ void block_scan(Scans &sh, double &mass, double &total)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    mass = wave_scan(mass);
    __syncthreads();
    if (lane == kWave - 1) sh.wave_sum[wave] = mass;
    __syncthreads();
    double before = 0.0;
    total = 0.0;
#pragma unroll 4
    for (int w = 0; w < kWaves; ++w) {
        if (w == wave) before = total;
        total += sh.wave_sum[w];
    }
    mass += before;
}
// the first thread for which `here` holds, or else the last for which `other` does (-1: none)
__device__ __forceinline__ int block_first(Scans &sh, bool here, bool other)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const uint64_t a = __ballot(here), b = __ballot(other);
    __syncthreads();
    if (lane == 0) sh.wave_mass[wave] = a, sh.wave_sum[wave] = __longlong_as_double((long long)b);
    __syncthreads();
    for (int w = 0; w < kWaves; ++w)
        if (sh.wave_mass[w]) return w * kWave + __builtin_ctzll(sh.wave_mass[w]);
    for (int w = kWaves - 1; w >= 0; --w) {
        const uint64_t bits = (uint64_t)__double_as_longlong(sh.wave_sum[w]);
        if (bits) return w * kWave + 63 - __builtin_clzll(bits);
    }
    return -1;
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
            for (int k = 0; k < kEpv; ++k) f[k] = e + k < V ? load_elem<DT>(p, e + k) : -kInf;
        }
    }
    // f(values, first entry, block) of every 64 vectors of the row, a wavefront each
    template <typename F>
    __device__ __forceinline__ void each(F f) const
    {
#pragma unroll 1
        for (int b = threadIdx.x / kWave; b < blocks; b += kWaves)
#pragma unroll 1
            for (int s = 0; s < steps; ++s) {
                float v[kEpv];
                const int64_t e = first(b, s);
                load(e, v);
                f(v, e, b);
            }
    }
};

// what is written for the token v, x being its logit less the maximum over the temperature; sums are in units of 2^-shift
__device__ __forceinline__ void tell(const SampleArgs &a, int64_t t, int64_t v, double x, double kept_mass, double full_mass, uint32_t kept)
{
    const double unit = a.shift * 0.69314718055994530942;
    a.token[t] = (int32_t)v;
    if (a.logp) a.logp[t] = (float)(x - (log(kept_mass) - unit));
    if (a.logp_full) a.logp_full[t] = (float)(x - (log(full_mass) - unit));
    if (a.kept) a.kept[t] = (int32_t)kept;
}

// All passes over a row that its lists do not settle.
template <typename DT>
struct Passes {
    static constexpr int EPV = DT::kPerVec;
    const SampleArgs &a;
    Shared &sh;
    Row<DT> row;
    Weigh weigh;

    // counts and masses of the entries whose key's bits above shift + bits are `prefix`, by their next `bits`
    __device__ void histogram(uint32_t prefix, int shift, int bits)
    {
        __syncthreads();
        for (int i = threadIdx.x; i < kBins; i += kThreads) sh.key.mass[i] = 0, sh.key.count[i] = 0;
        __syncthreads();
        const uint32_t mask = (1u << bits) - 1;
        row.each([&](const float *v, int64_t, int) {
#pragma unroll
            for (int k = 0; k < EPV; ++k) {
                const uint32_t key = key_of(v[k]);
                if (key > kKeyOfNegInf && (bits + shift == 32 || key >> (shift + bits) == prefix)) {
                    const uint32_t d = key >> shift & mask;
                    atomicAdd(&sh.key.count[d], 1u);
                    atomicAdd(reinterpret_cast<unsigned long long *>(&sh.key.mass[d]), (unsigned long long)weigh.whole(v[k]));
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
        uint64_t ms = 0;
        uint32_t cs = 0;
        const int top = kBins - 1 - (int)threadIdx.x * kEach;
#pragma unroll
        for (int i = 0; i < kEach; ++i) ms += sh.key.mass[top - i], cs += sh.key.count[top - i];
        uint64_t mi = ms;
        uint32_t ci = cs;
        block_scan(sh, mi, ci, mass_total, count_total);
        uint64_t ma = mass + mi - ms;
        uint32_t ca = count + ci - cs;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint64_t m = sh.key.mass[top - i];
            const uint32_t c = sh.key.count[top - i];
            if (MASS ? ma < target && ma + m >= target : ca < target && (uint64_t)ca + c >= target)
                sh.found_digit = top - i, sh.found_mass = ma, sh.found_count = ca;
            ma += m, ca += c;
        }
        __syncthreads();
        mass = sh.found_mass, count = sh.found_count;
        return sh.found_digit;
    }
    // the index of the n-th entry, from 1 on, that has this key
    __device__ int32_t index_of(uint32_t key, uint32_t n)
    {
        const int tid = threadIdx.x, lane = tid & (kWave - 1);
        __syncthreads();
        sh.block_count[tid] = 0;
        __syncthreads();
        row.each([&](const float *v, int64_t, int b) {
            int equal = 0;
#pragma unroll
            for (int k = 0; k < EPV; ++k) equal += __popcll(__ballot(key_of(v[k]) == key));
            if (lane == 0 && equal) sh.block_count[b] += equal;
        });
        __syncthreads();
        const uint32_t own = sh.block_count[tid];
        uint64_t m = 0, mt;
        uint32_t upto = own, ct;
        block_scan(sh, m, upto, mt, ct);
        if (upto >= n && upto - own < n) sh.found_digit = tid, sh.found_count = n - (upto - own);
        __syncthreads();
        if (tid < kWave) {
            const int b = (int)sh.found_digit;
            uint32_t left = sh.found_count;
            for (int s = 0; s < row.steps; ++s) {
                float v[EPV];
                const int64_t e = row.first(b, s);
                row.load(e, v);
                uint32_t equal = 0;
#pragma unroll
                for (int k = 0; k < EPV; ++k) equal += key_of(v[k]) == key ? 1u : 0u;
                const uint32_t scan = wave_scan(equal);
                if (scan >= left && scan - equal < left) {
                    uint32_t at = scan - equal;
#pragma unroll
                    for (int k = 0; k < EPV; ++k)
                        if (key_of(v[k]) == key && ++at == left) sh.found.last = (int32_t)(e + k);
                }
                const uint32_t all = __shfl(scan, kWave - 1, kWave);
                if (all >= left) break;
                left -= all;
            }
        }
        __syncthreads();
        return sh.found.last;
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
        const uint32_t equal = sh.key.count[digit];
        const uint64_t each = sh.key.mass[digit] / equal;  // (equal logits have equal weights)
        uint64_t ties = MASS ? (target - above + each - 1) / (each ? each : 1) : target - count;
        if (ties > equal) ties = equal;
        mass = above + ties * each;
        return Border{prefix, ties == equal ? kAnyIndex : index_of(prefix, (uint32_t)ties)};
    }
    // the border of top_k and top_p
    __device__ Border cut(const Policy &policy)
    {
        Border border{kKeyOfNegInf, -1};
        if (!policy.by_k && !policy.by_p) return border;
        histogram(0, 20, 12);
        uint64_t mass = 0, total;
        uint32_t count = 0, finite;
        find<true>(1, mass, count, total, finite);
        if (policy.by_k && policy.k < finite) {
            border = select<false>((uint64_t)policy.k, total);
            if (policy.by_p) histogram(0, 20, 12);
        }
        if (policy.by_p) {
            const double need = ceil((double)fmaxf(policy.p, 0.0f) * (double)total);
            uint64_t target = need < 1.0 ? 1 : (uint64_t)need;
            if (target > total) target = total;
            border = tighter(border, select<true>(target, mass));
        }
        return border;
    }
    // bits of the kept, and the token
    __device__ void finish(const Policy &policy, Border border, int64_t t, float top)
    {
        const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
        __syncthreads();
        sh.block_mass[tid] = 0;
        __syncthreads();
        uint64_t full = 0;
        uint32_t mine = 0;
#pragma unroll 1
        for (int b = wave; b < row.blocks; b += kWaves) {
            uint64_t in_block = 0;
#pragma unroll 1
            for (int s = 0; s < row.steps; ++s) {
                float v[EPV];
                const int64_t e = row.first(b, s);
                row.load(e, v);
                uint32_t bits = 0;
#pragma unroll
                for (int i = 0; i < EPV; ++i) {
                    const uint64_t w = weigh.whole(v[i]);
                    const bool keep = border.keeps(v[i], (int32_t)(e + i));
                    full += w;
                    in_block += keep ? w : 0;
                    bits |= (keep ? 1u : 0u) << i;
                }
                mine += __popc(bits);
                if (a.allowed) {
                    uint32_t word = bits << (e & 31);
#pragma unroll
                    for (int off = 1; off < 32 / EPV; off <<= 1) word |= __shfl_xor(word, off, kWave);
                    if ((e & 31) == 0 && e < a.V) a.allowed[t * a.allowed_ld + (e >> 5)] = (int32_t)word;
                }
            }
            const uint64_t sum = wave_sum((unsigned long long)in_block);
            if (lane == 0) sh.block_mass[b] = sum;
        }
        uint64_t full_total, total;
        uint32_t kept, none, zero = 0;
        block_scan(sh, full, mine, full_total, kept);
        __syncthreads();
        const uint64_t own = sh.block_mass[tid];
        uint64_t mass = own;
        block_scan(sh, mass, zero, total, none);
        // the block, then the entry, in whose part of the sum the number falls
        const uint64_t target = (uint64_t)((double)policy.u * (double)total);
        if (mass > target && mass - own <= target) sh.found_digit = tid, sh.found_mass = target - (mass - own);
        __syncthreads();
        if (wave != 0) return;
        const int b = (int)sh.found_digit;
        uint64_t left = sh.found_mass;
#pragma unroll 1
        for (int s = 0; s < row.steps; ++s) {
            float v[EPV];
            const int64_t e = row.first(b, s);
            row.load(e, v);
            uint64_t sum = 0;
#pragma unroll
            for (int i = 0; i < EPV; ++i) sum += border.keeps(v[i], (int32_t)(e + i)) ? weigh.whole(v[i]) : 0;
            const uint64_t upto = wave_scan((unsigned long long)sum);
            if (upto > left && upto - sum <= left) {
                uint64_t at = upto - sum;
                bool done = false;
#pragma unroll
                for (int i = 0; i < EPV; ++i) {
                    at += border.keeps(v[i], (int32_t)(e + i)) ? weigh.whole(v[i]) : 0;
                    if (!done && at > left) {
                        done = true;
                        tell(a, t, e + i, ((double)v[i] - (double)top) / (double)policy.tau, (double)total, (double)full_total, kept);
                    }
                }
            }
            if (__any(upto > left)) break;
            left -= __shfl((unsigned long long)upto, kWave - 1, kWave);
        }
    }
};

// The gathered entries.  Positions are in the order of the indices.
struct Lists {
    Shared &sh;
    const Weigh &weigh;
    uint32_t n;

    __device__ __forceinline__ int bin_of(float v, float top, float scale) const
    {
        return (int)fminf(fmaxf((top - v) * scale, 0.0f), (float)(kThreads - 1));
    }
    // the last entry that is kept: in bin found_digit, before which there are found_mass and found_count; false: too many there
    template <bool MASS>
    __device__ bool resolve(uint64_t target, float top, float scale, Border &border, uint64_t &mass) const
    {
        const int tid = threadIdx.x;
        const int bin = (int)sh.found_digit;
        const uint64_t mass_before = sh.found_mass;
        const uint32_t count_before = sh.found_count;
        if (sh.list.bin_count[bin] > kThreads) return false;  // (the same for all)
        uint32_t *at = sh.block_count;
        uint64_t *weight = sh.block_mass;
        if (tid == 0) sh.gathered = 0;
        __syncthreads();
        for (uint32_t i = tid; i < n; i += kThreads) {
            const float v = sh.list.value[i];
            if (bin_of(v, top, scale) == bin) {
                const uint32_t to = atomicAdd(&sh.gathered, 1u);
                at[to] = i;
                weight[to] = weigh.whole(v);
            }
        }
        __syncthreads();
        const uint32_t m = sh.gathered;
        if ((uint32_t)tid < m) {
            const uint32_t mine = at[tid];
            const float v = sh.list.value[mine];
            uint64_t ahead = mass_before;
            uint32_t before = count_before;
            for (uint32_t q = 0; q < m; ++q) {
                const float o = sh.list.value[at[q]];
                const bool first = o > v || (o == v && at[q] < mine);
                ahead += first ? weight[q] : 0;
                before += first ? 1u : 0u;
            }
            if (MASS ? ahead < target && ahead + weight[tid] >= target : before + 1 == target)
                sh.found = Border{key_of(v), sh.list.index[mine]}, sh.found_mass = ahead + weight[tid];
        }
        __syncthreads();
        border = sh.found;
        mass = sh.found_mass;
        return true;
    }
};

__device__ __forceinline__ void tell_none(const SampleArgs &a, int64_t t, bool bad)
{
    if (a.allowed)
        for (int64_t w = threadIdx.x; w < (a.V + 31) / 32; w += kThreads) a.allowed[t * a.allowed_ld + w] = 0;
    if (threadIdx.x == 0) {
        const float none = bad ? __builtin_nanf("") : -kInf;
        a.token[t] = -1;
        if (a.logp) a.logp[t] = none;
        if (a.logp_full) a.logp_full[t] = none;
        if (a.kept) a.kept[t] = 0;
    }
}
__device__ __forceinline__ float number_of(const Policy &policy) { return fminf(fmaxf(policy.u, 0.0f), 1.0f - 5.9604645e-8f); }
// the smallest float at or above max + temperature ln(min_p)
__device__ __forceinline__ float least_of(const Policy &policy, float top)
{
    const double least = (double)top + (double)policy.tau * log((double)fminf(policy.min_p, 1.0f));
    const float zt = (float)least;
    return (double)zt < least ? nextafterf(zt, kInf) : zt;
}

// The entry of a part in whose part of the kept sum the number falls; `within`: what of it lies in the part, in units of 2^-shift of
// the weight of weigh's maximum.
template <typename DT>
__device__ __forceinline__ void draw_in_part(const SampleArgs &a, Scans &sh, const Row<DT> &row, const Weigh &weigh, int part, double within,
                                             Border border, int64_t t, float top, float tau, double kept_mass, double full, uint32_t kept)
{
    constexpr int kEach = kSamplePart / kThreads;
    const int tid = threadIdx.x;
    const int64_t e = (int64_t)part * kSamplePart + tid * kEach;
    float v[kEach];
    double w[kEach], sum = 0.0;
#pragma unroll
    for (int k = 0; k < kEach; k += Row<DT>::kEpv) row.load(e + k, v + k);
#pragma unroll
    for (int k = 0; k < kEach; ++k) w[k] = border.keeps(v[k], (int32_t)(e + k)) ? weigh(v[k]) : 0.0, sum += w[k];
    double scan = sum, all;
    block_scan(sh, scan, all);
    const int thread = block_first(sh, scan > within && sum > 0.0, sum > 0.0);
    if (tid == thread) {
        double at = scan - sum;
        int64_t token = -1;
        double x = 0.0;
        bool done = false;
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            at += w[k];
            if (!done && w[k] > 0.0) token = e + k, x = (double)v[k], done = at > within;
        }
        tell(a, t, token, (x - (double)top) / (double)tau, kept_mass, full, kept);
    }
}

template <typename DT>
__global__ __launch_bounds__(kThreads) void sample_rows_kernel(SampleArgs a, int64_t row0, int64_t rows)
{
    __shared__ Scans sh;
    __shared__ int part_place[kThreads];
    __shared__ uint32_t part_bins[kThreads];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    if (tid < 32) sh.table[tid] = ldexp(kTable[tid], a.shift);
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const int64_t t = row0 + r;
        const SamplePart *part = a.part + r * a.parts;
        // ---- what the parts say together; a thread's own part where there is one for each
        float top = -kInf;
        SamplePart mine = {};
        mine.max = -kInf;
        bool bad = false;
        int far = 0;
        for (int q = tid; q < a.parts; q += kThreads) {
            mine = part[q];
            top = fmaxf(top, mine.max), bad |= mine.max != mine.max;
            far |= mine.max > -kInf && mine.place == kSampleFar;
        }
        top = wave_max(top);
        if (__any(bad)) top = __builtin_nanf("");
        __syncthreads();  // (the row before this one is done with everything)
        if (lane == 0) sh.wave_top[wave] = top;
        const bool any_far = __syncthreads_or(far);
        bad = false;
#pragma unroll 4
        for (int w = 0; w < kWaves; ++w) bad |= sh.wave_top[w] != sh.wave_top[w], top = fmaxf(top, sh.wave_top[w]);
        const Policy policy(a, t);
        bad |= policy.bad;
        SampleRow out = {};
        out.top = top;
        out.mode = kSampleDone;
        if (bad || top == -kInf) {
            tell_none(a, t, bad);
            if (tid == 0) a.row[r] = out;
            continue;
        }
        const bool each_part = a.parts <= kThreads;
        if (!policy.cut() && each_part && !a.allowed) {
            // ---- uncut: the part, then the entry, in whose part of the sum the number falls
            const double unit = kUnit / (double)policy.tau;
            const Weigh weigh{(double)top, unit, sh.table};
            double upto = mine.mass * weigh(mine.max), full;
            const double own = upto;
            block_scan(sh, upto, full);
            const double target = (double)number_of(policy) * full;
            const int chosen = block_first(sh, upto > target && own > 0.0, own > 0.0);
            __syncthreads();
            if (tid == chosen) sh.wave_sum[0] = fmax(target - (upto - own), 0.0) / weigh(mine.max), sh.wave_top[0] = mine.max;
            __syncthreads();
            const double within = sh.wave_sum[0] * ldexp(1.0, a.shift);
            const Weigh here{(double)sh.wave_top[0], unit, sh.table};
            uint64_t none = 0, none_total;
            uint32_t finite = mine.count, kept = 0;
            if (a.kept) block_scan(sh, none, finite, none_total, kept);
            const Row<DT> row{reinterpret_cast<const char *>(a.z) + t * a.ld * DT::kBytes, a.V, a.steps, a.blocks};
            draw_in_part(a, sh, row, here, chosen, within, Border{kKeyOfNegInf, -1}, t, top, policy.tau, full, full, kept);
            if (tid == 0) a.row[r] = out;
            continue;
        }
        out.mode = kSamplePasses;
        if (policy.cut() && each_part && !any_far) {
            // ---- cut: all parts' bins on the row's grid, a bin a thread
            const double grid = kGrid / (double)policy.tau;
            out.place = place_of(top, grid);
            if (tid < a.parts) part_place[tid] = mine.max > -kInf ? mine.place : kSampleFar, part_bins[tid] = mine.max > -kInf ? mine.bins : 0;
            __syncthreads();
            uint64_t sum = 0;
            uint32_t own_count = 0;
#pragma unroll 8
            for (int q = 0; q < a.parts; ++q) {
                const uint32_t b = (uint32_t)tid - ((uint32_t)out.place - (uint32_t)part_place[q]);
                if (b < part_bins[q]) {
                    const uint64_t v = a.bins[(r * a.parts + q) * kSampleBins + b];
                    sum += v & kWeightMask, own_count += (uint32_t)(v >> kWeightBits);
                }
            }
            // in units of the weight in the middle of bin 0, times 2^36: bins of 16 a power of two (even places of the table)
            const int down = (tid + 15) >> 4;
            const double own = (double)sum * ldexp(kTable[2 * (down * 16 - tid)], -down);
            double upto = own, all, tails = 0.0;
            block_scan(sh, upto, all);
            if (tid < a.parts && mine.max > -kInf) tails = mine.mass * exp2(-0.0625 * (double)(out.place - mine.place)) * 68719476736.0;
            double none = tails, tail;
            block_scan(sh, none, tail);
            uint64_t unused = 0, unused_total;
            uint32_t count = own_count, binned, finite = tid < a.parts ? mine.count : 0, all_finite;
            block_scan(sh, unused, count, unused_total, binned);
            unused = 0;
            block_scan(sh, unused, finite, unused_total, all_finite);
            out.full = all + tail;
            // ---- the bin of the tightest border; several may share it.  (The first kSampleBins hold all entries of every part.)
            const bool whole = tid < kSampleBins;
            const bool by_k = policy.by_k && policy.k < (int64_t)all_finite;
            const double need = (double)fmaxf(policy.p, 0.0f) * out.full;
            int bin_k = -1, bin_p = -1, bin_min = -1;
            bool lost = false;
            if (by_k) bin_k = block_first(sh, whole && (int64_t)count >= policy.k, false), lost |= bin_k < 0;
            if (policy.by_p && !by_k) bin_p = block_first(sh, whole && own_count > 0 && upto >= need, false), lost |= bin_p < 0;
            if (policy.by_min) {
                const float zt = least_of(policy, top);
                const int64_t b = (int64_t)out.place - place_of(zt, grid);
                bin_min = b < kSampleBins ? (int)b : kSampleBins;
            }
            int bin = kSampleAll;
            if (bin_k >= 0) bin = bin_k;
            if (bin_p >= 0) bin = bin_p;
            // (top_p is a share of what top_k leaves, so with both all of that is needed)
            if (bin_min >= 0 && bin_min < bin && !(by_k && policy.by_p)) bin = bin_min;
            if (bin == kSampleBins) bin = kSampleAll, lost |= all_finite > kSampleListed;
            // how many there are down to it, and in it
            if (tid == 0) sh.found_count = all_finite, sh.found_digit = 0, sh.wave_sum[0] = 0.0;
            __syncthreads();
            if (tid == bin) sh.found_count = count, sh.found_digit = own_count, sh.wave_sum[0] = upto - own;
            __syncthreads();
            const uint32_t down_to = sh.found_count, in_bin = sh.found_digit;
            out.bin = bin;
            out.above = sh.wave_sum[0];
            out.count = down_to - in_bin;
            out.share = policy.by_p && bin_p == bin ? need : -1.0;
            out.rank = bin_k == bin && bin_k >= 0 ? policy.k - out.count : -1;
            out.by_k = by_k;
            if (!lost) {
                if (down_to <= kSampleListed) out.mode = kSampleFew;
                else if (bin != kSampleAll && in_bin <= kSampleListed && !(by_k && policy.by_p)) out.mode = kSampleBin;
            }
        }
        if (tid == 0) a.row[r] = out;
    }
}

template <typename DT>
__global__ __launch_bounds__(kThreads) void sample_finish_kernel(SampleArgs a, int64_t row0, int64_t rows)
{
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    if (tid < 32) sh.table[tid] = ldexp(kTable[tid], a.shift);
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const int64_t t = row0 + r;
        const SampleRow row = a.row[r];
        if (row.mode == kSampleDone) continue;
        __syncthreads();  // (the table is there; the row before this one is done with everything)
        Policy policy(a, t);
        policy.u = number_of(policy);
        const float top = row.top;
        const Weigh weigh{(double)top, kUnit / (double)policy.tau, sh.table};
        const Row<DT> data{reinterpret_cast<const char *>(a.z) + t * a.ld * DT::kBytes, a.V, a.steps, a.blocks};
        Border border{kKeyOfNegInf, -1};
        if (policy.by_min) {
            const float zt = least_of(policy, top);
            if (zt > -kInf) border = Border{key_of(zt), kAnyIndex};
        }
        bool settled = row.mode != kSamplePasses;
        // what one unit of the bins' sums (2^-36 of the middle of bin 0) is in units of 2^-shift of the largest weight
        const double grid = kGrid / (double)policy.tau;
        const double to_whole = settled ? ldexp(exp2(((double)row.place - (double)top * grid) * 0.0625), a.shift - 36) : 0.0;
        const double full = row.full * to_whole;
        SampleSegment segment = {};
        uint32_t n = 0, place = 0;  // entries; where this thread's part's begin
        if (settled) {
            // ---- the gathered entries, in the order of the parts
            if (tid < a.parts) segment = a.segment[r * a.parts + tid];
            uint64_t none = 0, none_total;
            place = segment.listed;
            block_scan(sh, none, place, none_total, n);
            place -= segment.listed;
            if (tid < a.parts) sh.block_count[tid] = place;
            __syncthreads();
            for (int q = wave; q < a.parts; q += kWaves) {
                const SampleSegment &from = a.segment[r * a.parts + q];
                const uint32_t to = sh.block_count[q], many = from.listed;
                const uint2 *list = a.list + r * kSampleListed + from.start;
                for (uint32_t i = lane; i < many; i += kWave) {
                    const uint2 v = list[i];
                    sh.list.value[to + i] = __uint_as_float(v.x), sh.list.index[to + i] = (int32_t)v.y;
                }
            }
            const bool few = row.mode == kSampleFew;
            const bool by_k = few ? row.by_k : row.rank > 0, by_p = few ? policy.by_p : row.share >= 0.0;
            if (by_k || by_p) {
                // by logit, in bins between the largest and the smallest of them
                const Lists lists{sh, weigh, n};
                __syncthreads();
                float highest = -kInf, lowest = kInf;
                for (uint32_t i = tid; i < n; i += kThreads) highest = fmaxf(highest, sh.list.value[i]), lowest = fminf(lowest, sh.list.value[i]);
                highest = wave_max(highest), lowest = -wave_max(-lowest);
                if (lane == 0) sh.wave_top[wave] = highest, sh.wave_count[wave] = __float_as_uint(lowest);
                sh.list.bin_mass[tid] = 0, sh.list.bin_count[tid] = 0;
                __syncthreads();
#pragma unroll 4
                for (int w = 0; w < kWaves; ++w) highest = fmaxf(highest, sh.wave_top[w]), lowest = fminf(lowest, __uint_as_float(sh.wave_count[w]));
                const float scale = lowest < highest ? (float)(kThreads - 1) / (highest - lowest) : 0.0f;
                for (uint32_t i = tid; i < n; i += kThreads) {
                    const float v = sh.list.value[i];
                    const int b = lists.bin_of(v, highest, scale);
                    atomicAdd(&sh.list.bin_count[b], 1u);
                    atomicAdd(reinterpret_cast<unsigned long long *>(&sh.list.bin_mass[b]), (unsigned long long)weigh.whole(v));
                }
                __syncthreads();
                const uint64_t own = sh.list.bin_mass[tid];
                const uint32_t own_count = sh.list.bin_count[tid];
                uint64_t mass = own, list_mass;
                uint32_t count = own_count, list_count;
                block_scan(sh, mass, count, list_mass, list_count);
                double total = full;  // of what top_p is a share of
                const int64_t k = few ? policy.k : row.rank;
                if (by_k && k <= (int64_t)list_count) {
                    if ((int64_t)count >= k && (int64_t)(count - own_count) < k)
                        sh.found_digit = tid, sh.found_mass = mass - own, sh.found_count = count - own_count;
                    __syncthreads();
                    Border here;
                    uint64_t left;
                    settled = lists.resolve<false>((uint64_t)k, highest, scale, here, left);
                    if (settled) border = tighter(border, here), total = (double)left;
                    __syncthreads();
                }  // (else min_p ends the list before the k-th, and there is no top_p)
                if (settled && by_p) {
                    const double need = ceil(few ? (double)fmaxf(policy.p, 0.0f) * total : (row.share - row.above) * to_whole);
                    uint64_t target = need < 1.0 ? 1 : (uint64_t)need;
                    if (target > list_mass) target = list_mass;
                    if (mass >= target && mass - own < target)
                        sh.found_digit = tid, sh.found_mass = mass - own, sh.found_count = count - own_count;
                    __syncthreads();
                    Border here;
                    uint64_t left;
                    settled = lists.resolve<true>(target, highest, scale, here, left);
                    if (settled) border = tighter(border, here);
                }
            }
            __syncthreads();
        }
        if (settled) {
            // ---- the kept of the gathered: in the order of their indices, so many a thread
            const int each = (int)((n + kThreads - 1) / kThreads);
            uint64_t sum = 0;
            uint32_t kept = 0;
            for (int i = 0; i < each; ++i) {
                const uint32_t q = tid * each + i;
                if (q < n && border.keeps(sh.list.value[q], sh.list.index[q])) sum += weigh.whole(sh.list.value[q]), ++kept;
            }
            uint64_t scan = sum, total;
            uint32_t kept_total;
            block_scan(sh, scan, kept, total, kept_total);
            if (row.mode == kSampleBin) {
                // ---- each part's kept: what is above the bin, and of the bin what is in its segment
                if (tid < a.parts) sh.block_count[tid] = place;
                __syncthreads();
                for (int q = wave; q < a.parts; q += kWaves) {
                    const uint32_t to = sh.block_count[q], many = a.segment[r * a.parts + q].listed;
                    uint64_t in_part = 0;
                    for (uint32_t i = lane; i < many; i += kWave)
                        if (border.keeps(sh.list.value[to + i], sh.list.index[to + i])) in_part += weigh.whole(sh.list.value[to + i]);
                    in_part = wave_sum((unsigned long long)in_part);
                    if (lane == 0) sh.block_mass[q] = in_part;
                }
                __syncthreads();
                const double own = tid < a.parts ? segment.above * to_whole + (double)sh.block_mass[tid] : 0.0;
                double upto = own, mass;
                block_scan(sh, upto, mass);
                const double target = (double)policy.u * mass;
                const int chosen = block_first(sh, upto > target && own > 0.0, own > 0.0);
                __syncthreads();
                if (tid == chosen) sh.wave_sum[0] = fmax(target - (upto - own), 0.0);
                __syncthreads();
                const double within = sh.wave_sum[0];
                draw_in_part(a, sh, data, weigh, chosen, within, border, t, top, policy.tau, mass, full, row.count + kept_total);
                if (a.allowed) {
                    // (entries above the bin, and the border's part of it: what the border says of every entry)
                    constexpr int EPV = DT::kPerVec;
                    data.each([&](const float *v, int64_t e, int) {
                        uint32_t word = 0;
#pragma unroll
                        for (int k = 0; k < EPV; ++k) word |= (border.keeps(v[k], (int32_t)(e + k)) ? 1u : 0u) << k;
                        word <<= e & 31;
#pragma unroll
                        for (int off = 1; off < 32 / EPV; off <<= 1) word |= __shfl_xor(word, off, kWave);
                        if ((e & 31) == 0 && e < a.V) a.allowed[t * a.allowed_ld + (e >> 5)] = (int32_t)word;
                    });
                }
                continue;
            }
            // ---- few: the entry in whose part of the sum the number falls
            const uint64_t target = (uint64_t)((double)policy.u * (double)total);
            if (scan > target && scan - sum <= target) {
                uint64_t at = scan - sum;
                for (int i = 0; i < each; ++i) {
                    const uint32_t q = tid * each + i;
                    const float v = sh.list.value[q];
                    if (border.keeps(v, sh.list.index[q])) at += weigh.whole(v);
                    if (at > target) {
                        tell(a, t, sh.list.index[q], ((double)v - (double)top) / (double)policy.tau, (double)total, full, kept_total);
                        break;
                    }
                }
            }
            if (a.allowed) {
                // bits of so many words at a time
                constexpr int kWords = 2 * kSampleBlocks;
                uint32_t *words = reinterpret_cast<uint32_t *>(sh.block_mass);
                const int64_t all = (a.V + 31) / 32;
                for (int64_t begin = 0; begin < all; begin += kWords) {
                    __syncthreads();
                    words[tid] = 0, words[tid + kThreads] = 0;
                    __syncthreads();
                    for (uint32_t q = tid; q < n; q += kThreads) {
                        const int32_t e = sh.list.index[q];
                        const int64_t w = (e >> 5) - begin;
                        if (w >= 0 && w < kWords && border.keeps(sh.list.value[q], e)) atomicOr(&words[w], 1u << (e & 31));
                    }
                    __syncthreads();
                    for (int64_t w = tid; w < kWords && begin + w < all; w += kThreads) a.allowed[t * a.allowed_ld + begin + w] = (int32_t)words[w];
                }
            }
            continue;
        }
        // ---- the row, as often as its cuts ask
        border = Border{kKeyOfNegInf, -1};
        if (policy.by_min) {
            const float zt = least_of(policy, top);
            if (zt > -kInf) border = Border{key_of(zt), kAnyIndex};
        }
        Passes<DT> passes{a, sh, data, weigh};
        passes.finish(policy, tighter(border, passes.cut(policy)), t, top);
    }
}

template <typename DT>
void launch(const SampleArgs &a, hipStream_t s)
{
    for (int64_t row0 = 0; row0 < a.T; row0 += kSampleRows) {
        const int64_t rows = a.T - row0 < kSampleRows ? a.T - row0 : kSampleRows, parts = rows * a.parts;
        const int grid = (int)(parts < (1 << 24) ? parts : 1 << 24);
        sample_parts_kernel<DT><<<grid, kPartThreads, 0, s>>>(a, row0, rows);
        sample_rows_kernel<DT><<<(int)rows, kThreads, 0, s>>>(a, row0, rows);
        // (rows that are all uncut are done; what is not known on the host, temperatures of 0 among it, may cut)
        if (!a.temperature && !a.top_k && !a.top_p && !a.min_p && !a.allowed && a.parts <= kThreads) continue;
        sample_gather_kernel<DT><<<grid, kPartThreads, 0, s>>>(a, row0, rows);
        sample_finish_kernel<DT><<<(int)rows, kThreads, 0, s>>>(a, row0, rows);
    }
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, hipStream_t s)
{
    if (a.dt == A3PO_F32) launch<F32>(a, s);
    else launch<Bf16>(a, s);
    return hipGetLastError();
}

}  // namespace a3po
