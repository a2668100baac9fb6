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
//            power of two of their weight (1/4 under top-k), on one grid for all parts, so that parts add up
//   rows:    uncut, the token: the part, then the entry, in whose part of the sum the drawn number falls.  Cut, the bin that the
//            border is in
//   gather:  the entries down to that bin, where they are few, else that bin's alone: parts without any are not read again
//   finish:  the border among those entries, and the token
// Cut rows that this does not settle are gone over by one workgroup as often as their cuts ask (passes): a border among more entries than
// can be listed (kSampleFewest down to it, or kSampleListed in its bin; with top-k and top-p the former), one 2^-32 below the largest weight
// (2^-128 under top-k), also where that leaves every entry, values off the grid; and all rows of more than 512 parts.
//
// Why parts: one row decodes alone as often as a thousand do together, so the row's passes are spread over as many compute units as it
// has parts, and a part stays in registers from its maximum to its bins.  Why bins on a grid of absolute places: parts need not know the
// row's maximum, and what they find adds up.  One read of the row is needed (38 MB of 64 x 151,936 fp32 logits take 8 us at a large
// copy's 4.9 TB/s), a second one of the parts that hold entries down to the border.
// Measured, us (all five or six kernels back to back; by kernel: parts / rows / gather / finish / rows with passes / bits):
//     1 x  32,000 fp32, top-p 0.95                         28 to 34   (7 / 6 / 6 / 11 / 3 to 4: five launches in a row, whose host time differs by call)
//    64 x 151,936 fp32, top-p 0.95                         64   (19 / 8 / 16 / 20 / 4)
//   300 x  50,001 fp32, top-k 50, top-p, min-p, bits       80   (29 / 8 / 20 / 18 / 5 / 4)
//   256 x 151,936 bf16, top-p 0.9 of flat rows, bits      136   (37 / 9 / 36 / 30 / 6 / 18)
//  1024 x 151,936 bf16, uncut                             113   (one pass over the rows 114, tokens 11; under the profiler)
//   1 / 64 / 512 x 151,936 fp32, uncut with bits          25 / 41 / 193   (parts, rows, bits; without bits 15 / 21 / 96)
// What bounds them: vector instructions where there are many parts (uncut 21 an entry, 9 of them in 64 bits: active in 94 % of a
// compute unit's busy cycles; parts of flat rows 26 an entry, 85 %), latencies in a row where there are few: a part's load, maximum, bins; a row's parts,
// scan, border; list, border, part, token.  Spilled registers: finish 10 in either type, passes 5 in fp32 and 47 in bfloat16, gather 2 in
// bfloat16, none elsewhere.
//
// In a bin, weights are relative to the bin's and added as whole numbers of 2^-36, their count above them in the same 64 bits: one
// atomic an entry.  Everywhere else that entries are counted by atomics weights are multiples of 2^-shift of the row's largest, so many that
// 64 bits hold the sum: shift = 62 - log2 V (50 at most) in passes, 48 at least among listed entries, of which there are fewer than
// 2^14.  Both make additions commute.  What that rounds: sums of listed entries and bins are within 2^-35 of the kept sum, those of passes
// within V 2^-(shift + 1) (151,936 entries 2^-27).  Uncut rows are summed in double, in one order.
#include "a3po_common.h"
#include "a3po_launch.h"

namespace a3po {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / kWave;
constexpr int kBins = 4096;
constexpr uint32_t kKeyOfNegInf = 0x007FFFFFu;
constexpr int kPartThreads = 256, kPartWaves = kPartThreads / kWave;
constexpr int kDirect = 128;  // gathered entries that are each compared with all others

constexpr float kInf = __builtin_huge_valf();
constexpr double kRound = 6755399441055744.0;   // 1.5 * 2^52: added to a number it leaves the whole number next to it in the low word
constexpr double kUnit = 46.166241308446828384;  // 32 log2(e)

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

// a b + c with c in scalar registers.  (The compiler takes v_fmac_f64, whose c is overwritten, and copies c first.)
__device__ __forceinline__ double fma_scalar(double a, double b, double c)
{
    double r;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "s"(c));
    return r;
}

// e^x: 2^(i / 32) from a table (one entry a pair of LDS banks: lanes never wait for one another), the rest of the exponent by a
// series whose first term left out, (ln 2 / 64)^6 / 720, is 2^-48
struct Weigh {
    double max, unit;     // unit: 32 log2(e) / temperature
    const double *table;  // 2^(i / 32) times what the result is to be scaled by
    // below 2^-1000 of the largest there is no weight (masked entries: also where the temperature is infinite, as -inf times 0 is NaN)
    __device__ __forceinline__ double operator()(float z) const { return has(z) ? floored(z) : 0.0; }
    __device__ __forceinline__ bool has(float z) const { return ((double)z - max) * unit >= -32000.0; }
    // (2^-1000 for those)
    __device__ __forceinline__ double floored(float z) const
    {
        constexpr double a1 = 0.69314718055994530942 / 32, a2 = a1 * a1 / 2, a3 = a2 * a1 / 3, a4 = a3 * a1 / 4, a5 = a4 * a1 / 5;
        const double y = fmax(((double)z - max) * unit, -32000.0);
        const double t = y + kRound;
        const int n = __double2loint(t);
        const double r = y - (t - kRound);
        const double b = table[n & 31];
        const double scale = __hiloint2double(__double2hiint(b) + ((n >> 5) << 20), __double2loint(b));
        return scale * fma(fma_scalar(fma_scalar(fma_scalar(fma_scalar(r, a5, a4), r, a3), r, a2), r, a1), r, 1.0);
    }
    __device__ __forceinline__ uint64_t whole(float z) const
    {
        return (uint64_t)__double_as_longlong(floored(z) + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
    }
};
// 2^(-b / 16)
__device__ __forceinline__ double down_by(int b)
{
    const int whole = (b + 15) >> 4;
    return ldexp(kTable[2 * (whole * 16 - b)], -whole);
}

// orders floats as whole numbers; -0 and 0 are one
__device__ __forceinline__ uint32_t key_of(float z)
{
    const uint32_t u = __float_as_uint(z + 0.0f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// (fmaxf makes a quiet NaN of each operand first, an instruction each; NaN is looked for apart)
__device__ __forceinline__ float max2(float a, float b)
{
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ float min3(float a, float b, float c)
{
    float r;
    asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// Sums over the lanes before and up to each: within rows of 16 lanes, then rows 1 and 3 take what ends row 0 and 2, then the upper
// half what ends the lower.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t lanes(uint32_t v)  // 0 where there is no such lane
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS, typename T>
__device__ __forceinline__ T from_lanes(T v)
{
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, lanes<CTRL, ROWS>(__builtin_bit_cast(uint32_t, v)));
    } else {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        return __builtin_bit_cast(T, (uint64_t)lanes<CTRL, ROWS>((uint32_t)(u >> 32)) << 32 | lanes<CTRL, ROWS>((uint32_t)u));
    }
}
template <typename T>
__device__ __forceinline__ T wave_scan(T v)  // inclusive
{
    v += from_lanes<0x111, 0xF>(v);
    v += from_lanes<0x112, 0xF>(v);
    v += from_lanes<0x114, 0xF>(v);
    v += from_lanes<0x118, 0xF>(v);
    v += from_lanes<0x142, 0xA>(v);
    return v + from_lanes<0x143, 0xC>(v);
}
template <typename T>
__device__ __forceinline__ T last_lane(T v)
{
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), kWave - 1));
    } else {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        return __builtin_bit_cast(T, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), kWave - 1) << 32 |
                                         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, kWave - 1));
    }
}
template <typename T>
__device__ __forceinline__ T wave_sum(T v)
{
    return last_lane(wave_scan(v));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float max_with(float v)
{
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), CTRL, ROWS, 0xF, false)));
}
__device__ __forceinline__ float wave_max(float v)
{
    v = max_with<0x111, 0xF>(v);
    v = max_with<0x112, 0xF>(v);
    v = max_with<0x114, 0xF>(v);
    v = max_with<0x118, 0xF>(v);
    v = max_with<0x142, 0xA>(v);
    return last_lane(max_with<0x143, 0xC>(v));
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

// What the row's arrays say, absent ones being neutral; a temperature of NaN where they say nothing that can be followed.
struct Policy {
    float tau, p, min_p, u;
    int64_t k;
    __device__ __forceinline__ Policy(const SampleArgs &a, int64_t t)
        : tau(a.temperature ? a.temperature[t] : 1.0f), p(a.top_p ? a.top_p[t] : 1.0f), min_p(a.min_p ? a.min_p[t] : 0.0f),
          u(a.uniform[t]), k(a.top_k ? a.top_k[t] : 0)
    {
        if (tau == 0.0f) tau = 1.0f, k = 1;
        if (!(tau >= 0.0f) || p != p || min_p != min_p || u != u) tau = __builtin_nanf("");
        if (k >= a.V) k = 0;
    }
    __device__ __forceinline__ bool bad() const { return tau != tau; }
    __device__ __forceinline__ bool by_k() const { return k > 0; }
    __device__ __forceinline__ bool by_p() const { return p < 1.0f; }
    __device__ __forceinline__ bool by_min() const { return min_p > 0.0f; }
    // Bins of 1/4 power of two instead of 1/16 reach four times as far: the k-th entry may be far below the largest.  (Rows with one entry
    // 40 ahead, top-k 50, 64 / 300 x 151,936 bf16: 47 / 109 us; with bins of 1/16, in passes, 179 / 282.)
    __device__ __forceinline__ int coarse() const { return by_k() ? 2 : 0; }
    __device__ __forceinline__ bool cut() const { return by_k() || by_p() || by_min(); }
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
    __device__ __forceinline__ void each(F f)
    {
#pragma unroll
        for (int v = 0; v < kVectors; ++v) {
            float x[EPV];
            asm volatile("" : "+v"(raw[v].x), "+v"(raw[v].y), "+v"(raw[v].z), "+v"(raw[v].w));  // (nothing of one pass is kept for the next)
            unpack<DT>(raw[v], x);
#pragma unroll
            for (int k = 0; k < EPV; ++k) f(x[k], v * EPV + k);
            __builtin_amdgcn_sched_barrier(0);  // (all vectors at once take more registers than they save time)
        }
    }
};

// Places on the grid: the whole number next to z times 16 log2(e) / temperature, by one rounding, so that larger logits never have
// smaller places.  `lowest` stands for everything that is further below than whole numbers of 32 bits reach.
constexpr double kNear = 1.0e9;
constexpr double kPlace = 2.0 / kUnit;  // what a place is of a temperature
__device__ __forceinline__ float lowest_of(float tau) { return (float)(-0.75e9 * kPlace * (double)tau); }
__device__ __forceinline__ int place_of(float z, double grid, float lowest) { return __double2loint(fma((double)max2(z, lowest), grid, kRound)); }
// the smallest float whose place is at least p; step: 1 / grid, nearly
__device__ __forceinline__ float first_at(int p, double grid, double step, float lowest)
{
    float z = (float)(((double)p - 0.5) * step);
#pragma unroll 1
    while (place_of(z, grid, lowest) >= p) z = nextafterf(z, -kInf);
#pragma unroll 1
    while (place_of(z, grid, lowest) < p) z = nextafterf(z, kInf);
    return z;
}
// in a bin's sum: the count in the upper 14 bits, weights times 2^36 below (the bin's middle is 1, its largest below 1.03, or 1.10 in bins of 1/4
// power of two: 8,192 of them are below 2^50)
constexpr int kWeightBits = 50;
constexpr uint64_t kWeightMask = (1ull << kWeightBits) - 1;
constexpr double kOne = 68719476736.0, kCounted = 5629499534213120.0;  // 2^36, 2^52 + 2^50

// The weights of an uncut part are 2^(z unit / 32) as they are: 64 bits hold 900 powers of two either way, and no maximum has to be
// known before.  Where the part's reaches further, or no float is far below it (temperatures from 1e28 on), they are relative to the
// maximum.  (The grid reaches further; see kNear.)
constexpr double kWide = 900.0 * 32;
__device__ __forceinline__ bool is_wide(float top, double unit) { return !(fabs((double)top * unit) < kWide && unit > 1e-27); }
__device__ __forceinline__ bool is_far(float top, double unit) { return !(fabs((double)top * unit) < kNear && unit > 1e-27); }

// NaN if either is
__device__ __forceinline__ float maximum(float a, float b)
{
    float r;
    asm("v_maximum3_f32 %0, %1, %2, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}

// One pass over an uncut part: the sum of the weights (NaN where an entry is NaN or +inf), the largest and the smallest logit.
template <typename DT>
__device__ __forceinline__ double sum_of(PartEntries<DT> &z, double unit, const double *table, float &top, float &low)
{
    constexpr double a1 = 0.69314718055994530942 / 32, a2 = a1 * a1 / 2, a3 = a2 * a1 / 3, a4 = a3 * a1 / 4, a5 = a4 * a1 / 5;
    // (a5 r^5 is replaced by the cubic next to it on [-1/2, 1/2]: off by a5 / 512 at most, 2^-43)
    constexpr double b3 = a3 + a5 * (5.0 / 16), b1 = a1 - a5 * (5.0 / 256);
    const float lowest = fmaxf((float)(-32000.0 / unit), -3.402823466e38f);
    double mass = 0.0;
    float last_one = 0.0f;
    top = -kInf, low = kInf;
    z.each([&](float x, int k) {
        if (k & 1) top = max3(top, last_one, x), low = min3(low, last_one, x);
        last_one = x;
        const double d = (double)maximum(x, lowest), n = fma(d, unit, kRound), q = fma(d, unit, -(n - kRound));
        const int whole = __double2loint(n);
        const double e = table[whole & 31];
        const double p = fma(fma(fma(fma(q, a4, b3), q, a2), q, b1), q, 1.0);
        mass = fma(__hiloint2double(__double2hiint(e) + (whole << 15), __double2loint(e)), p, mass);
        if (k % 4 == 3) asm volatile("" : "+v"(mass));  // (here, not where it is used)
    });
    return mass;
}

// What a part has found, written in one store: memory takes half a line's writing in two turns, and the next kernel waits for it.
union PartRecord {
    SamplePart part;
    uint32_t words[sizeof(SamplePart) / 4];
};
__device__ __forceinline__ void write_part(PartRecord &record, SamplePart &to, float top, int place, uint32_t bins, uint32_t count)
{
    if (threadIdx.x >= kWave) return;
    if (threadIdx.x == 0) record.part.max = top, record.part.place = place, record.part.bins = bins, record.part.count = count;
    // (lane 0's words are read by other lanes: this orders them within the wave, where LDS keeps its order by itself, for no instruction)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (threadIdx.x < sizeof(SamplePart) / 4) reinterpret_cast<uint32_t *>(&to)[threadIdx.x] = record.words[threadIdx.x];
}

// An uncut part: four waves that do not wait for one another until they have their sums.
template <typename DT>
__device__ __forceinline__ void sum_part(const SampleArgs &a, PartEntries<DT> &z, float tau, const double *table, PartRecord &record, float (&wave_top)[kPartWaves],
                                         uint32_t (&wave_count)[kPartWaves], SamplePart &to)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const double unit = kUnit / (double)tau;
    float top, low;
    double mass = wave_sum(sum_of(z, unit, table, top, low));
    top = wave_max(top), low = -wave_max(-low);
    bool bad = mass != mass || top == kInf;
    if (bad && top < kInf && is_wide(top, unit)) {  // (the sum says nothing)
        bad = false;
        z.each([&](float x, int) { bad |= x != x; });
        bad = __any(bad);
    }
    uint32_t count = 0;
    if (a.kept) {
        if (low > -kInf) count = kWave * PartEntries<DT>::kEach;  // (the same for all of the wave)
        else {
            z.each([&](float x, int) { count += x > -kInf ? 1u : 0u; });
            count = wave_sum(count);
        }
    }
    if (lane == 0) wave_top[wave] = bad ? __builtin_nanf("") : top, wave_count[wave] = count;
    __syncthreads();
    bool any_bad = false;
    const float own_top = top;
    top = -kInf, count = 0;
#pragma unroll
    for (int w = 0; w < kPartWaves; ++w) any_bad |= wave_top[w] != wave_top[w], top = fmaxf(top, wave_top[w]), count += wave_count[w];
    const Weigh weigh{(double)top, unit, kTable};
    if (!any_bad && top > -kInf && is_wide(top, unit)) {
        mass = 0.0;
        z.each([&](float x, int) {
            mass += weigh(x);
            asm volatile("" : "+v"(mass));
        });
        mass = wave_sum(mass);
    }
    // (a quarter has mass where one of its entries has a weight beside the part's largest: sum_of counts those without at its `lowest`, and a
    // drawn number of 0 would fall to them)
    if (lane == 0) record.part.mass[wave] = top > -kInf && weigh.has(own_top) ? mass : 0.0;
    __syncthreads();
    write_part(record, to, any_bad ? __builtin_nanf("") : top, kSampleFar, 0, count);
}

// Rows that the host knows to be uncut.
template <typename DT>
__global__ __launch_bounds__(kPartThreads, DT::kBytes == 4 ? 4 : 5) void sample_sums_kernel(SampleArgs a, int64_t row0, int64_t rows)
{
    __shared__ double table[32];
    __shared__ float wave_top[kPartWaves];
    __shared__ uint32_t wave_count[kPartWaves];
    __shared__ PartRecord record;
    const int tid = threadIdx.x;
    if (tid < 32) table[tid] = __hiloint2double(__double2hiint(kTable[tid]) - (tid << 15), __double2loint(kTable[tid]));
    for (int64_t i = blockIdx.x; i < rows * a.parts; i += gridDim.x) {
        const int64_t r = i / a.parts, t = row0 + r;
        const int64_t begin = (i - r * a.parts) * kSamplePart;
        PartEntries<DT> z;
        z.load(reinterpret_cast<const char *>(a.z) + (t * a.ld + begin) * DT::kBytes, (int)min(a.V - begin, (int64_t)kSamplePart));
        __syncthreads();  // (the table is there; the part before this one is done with the shared arrays)
        sum_part(a, z, 1.0f, table, record, wave_top, wave_count, a.part[i]);
    }
}

// A part: maximum, bins, what lies behind them.  256 threads hold 8,192 entries, 32 (fp32) or 16 (bfloat16) registers a thread.  Five
// workgroups a compute unit (flat rows 131 us for four's 134), three with fp32, where four spill 13 registers (64 x 151,936 70 us for 64).  Two
// sets of bins by even and odd lanes, against lanes that add to one bin, changed nothing (flat rows' parts 47.5 us for 46.9): instructions
// bound it, not the atomics.
template <typename DT>
__global__ __launch_bounds__(kPartThreads, DT::kBytes == 4 ? 3 : 5) void sample_parts_kernel(SampleArgs a, int64_t row0, int64_t rows)
{
    using Entries = PartEntries<DT>;
    __shared__ double table[32];
    __shared__ uint64_t bins[kSampleBins + kWave];
    __shared__ float wave_top[kPartWaves];
    __shared__ uint32_t wave_count[kPartWaves], wave_last[kPartWaves];
    __shared__ PartRecord record;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    // (with the exponent's share of 15 bits taken out, so that adding n << 15 puts the whole exponent in)
    if (tid < 32) table[tid] = __hiloint2double(__double2hiint(kTable[tid]) - (tid << 15), __double2loint(kTable[tid]));
    for (int64_t i = blockIdx.x; i < rows * a.parts; i += gridDim.x) {
        const int64_t r = i / a.parts, t = row0 + r;
        const int64_t begin = (i - r * a.parts) * kSamplePart;
        Entries z;
        z.load(reinterpret_cast<const char *>(a.z) + (t * a.ld + begin) * DT::kBytes, (int)min(a.V - begin, (int64_t)kSamplePart));
        const Policy policy(a, t);
        if (!policy.cut() && !policy.bad()) {
            __syncthreads();  // (the part before this one is done with the shared arrays)
            sum_part(a, z, policy.tau, table, record, wave_top, wave_count, a.part[i]);
            continue;
        }
        const double unit = kUnit / (double)policy.tau;
        float top = -kInf, low = kInf, last_one = 0.0f;
        bool bad = false;
        z.each([&](float x, int k) {
            // (two at a time)
            if (k & 1) top = max3(top, last_one, x), low = min3(low, last_one, x), bad |= __builtin_isunordered(x, last_one);
            last_one = x;
        });
        top = wave_max(top), low = -wave_max(-low);
        if (__any(bad) || top == kInf) top = __builtin_nanf("");
        __syncthreads();  // (the part before this one is done with the shared arrays)
        if (lane == 0) wave_top[wave] = top;
#pragma unroll
        for (int b = tid; b < kSampleBins; b += kPartThreads) bins[b] = 0;
        __syncthreads();
        bad = false, top = -kInf;
#pragma unroll
        for (int w = 0; w < kPartWaves; ++w) bad |= wave_top[w] != wave_top[w], top = fmaxf(top, wave_top[w]);
        if (bad || policy.bad() || top == -kInf) {  // (nothing to sum)
            if (tid == 0) {
                SamplePart out = {};
                out.max = bad ? __builtin_nanf("") : top;
                a.part[i] = out;
            }
            continue;
        }
        double mass = 0.0;
        uint32_t count = 0, bins_used = 0;
        int place = kSampleFar;
        const bool far = is_far(top, unit);
        if (!far) {
            const int coarse = policy.coarse();
            const double grid = unit * (coarse ? 0.125 : 0.5), step = kPlace * (double)policy.tau * (coarse ? 4.0 : 1.0);
            const float lowest = lowest_of(policy.tau);
            place = place_of(top, grid, lowest);
            const float behind = first_at(place - kSampleBins + 1, grid, step, lowest);  // the bins' smallest logit
            // Entry x's bin, the last ones first, or a place of the lane's own: without branches the entries' arithmetic overlaps.
            // w as it is in memory holds 4301 = 4 * 1075 + 1 where a bin's sum has its count, so N of them hold 4301 N modulo 2^14.
            const uint32_t base = 8u * (uint32_t)(kSampleBins - 1 - place), beside = 8u * (uint32_t)(kSampleBins + lane);
            auto put = [&](auto weigh) {
                z.each([&](float x, int) {
                    const double d = (double)x, n = fma(d, grid, kRound), q = fma(d, grid, -(n - kRound));
                    const double w = weigh(q);
                    const uint32_t at = ((uint32_t)__double2loint(n) << 3) + base;
                    atomicAdd(reinterpret_cast<unsigned long long *>(reinterpret_cast<char *>(bins) + (x >= behind ? at : beside)),
                              (unsigned long long)__double_as_longlong(w));
                });
            };
            // 2^(q / 16), 2^(q / 4): the series' last term, a5 q^5 or a7 q^7, is replaced by the polynomial next to it on [-1/2, 1/2], off by
            // a5 / 512 or a7 / 8192 at most, 2^-38 or 2^-43
            if (!coarse)
                put([](double q) {
                    constexpr double a1 = 0.69314718055994530942 / 16, a2 = a1 * a1 / 2, a3 = a2 * a1 / 3, a4 = a3 * a1 / 4, a5 = a4 * a1 / 5;
                    constexpr double b3 = a3 + a5 * (5.0 / 16), b1 = a1 - a5 * (5.0 / 256);
                    return fma_scalar(fma_scalar(fma_scalar(fma_scalar(q, a4 * kOne, b3 * kOne), q, a2 * kOne), q, b1 * kOne), q, kOne + kCounted);
                });
            else
                put([](double q) {
                    constexpr double a1 = 0.69314718055994530942 / 4, a2 = a1 * a1 / 2, a3 = a2 * a1 / 3, a4 = a3 * a1 / 4, a5 = a4 * a1 / 5, a6 = a5 * a1 / 6,
                                     a7 = a6 * a1 / 7;
                    constexpr double b5 = a5 + a7 * (7.0 / 16), b3 = a3 - a7 * (7.0 / 128), b1 = a1 + a7 * (7.0 / 4096);
                    const double high = fma_scalar(fma_scalar(fma_scalar(q, a6 * kOne, b5 * kOne), q, a4 * kOne), q, b3 * kOne);
                    return fma_scalar(fma_scalar(fma_scalar(high, q, a2 * kOne), q, b1 * kOne), q, kOne + kCounted);
                });
            // what lies behind the bins is below 2^-32 of the largest, all of it below 2^-19: what fp32 loses of that, 2^-18 of it, is
            // below 2^-37
            if (low < behind) {
                const float scale = (float)(unit * 0.03125), shift = (float)(fma((double)top, grid, -(double)place) * (coarse ? 0.25 : 0.0625));
                float tail = 0.0f;
                z.each([&](float x, int k) {
                    tail += x < behind ? exp2_hw(fmaf(x - top, scale, shift)) : 0.0f;
                    if (k % 4 == 3) asm volatile("" : "+v"(tail));
                });
                mass = (double)tail;
            }
            __syncthreads();  // (the bins are whole)
#pragma unroll
            for (int b = tid; b < kSampleBins; b += kPartThreads) {
                uint64_t sum = bins[kSampleBins - 1 - b];
                sum = (sum & kWeightMask) | (uint64_t)((uint32_t)(sum >> kWeightBits) * 7173u & 0x3FFFu) << kWeightBits;  // 1 / 4301 modulo 2^14
                bins[kSampleBins - 1 - b] = sum;
                if (sum) bins_used = b + 1;
                const int e = b << policy.coarse();
                const double middle = table[-2 * e & 31];  // 2^(-e / 16)
                mass = fma((double)(sum & kWeightMask) * (1.0 / kOne), __hiloint2double(__double2hiint(middle) - (e << 16), __double2loint(middle)), mass);
            }
        }
        if (low > -kInf) count = Entries::kEach;  // (the same for all of the wave)
        else z.each([&](float x, int) { count += x > -kInf ? 1u : 0u; });
        mass = wave_sum(mass);
        count = wave_sum(count);
        bins_used = (uint32_t)wave_max((float)bins_used);
        if (lane == 0) record.part.mass[wave] = mass, wave_count[wave] = count, wave_last[wave] = bins_used;
        __syncthreads();
        count = bins_used = 0;
#pragma unroll
        for (int w = 0; w < kPartWaves; ++w) count += wave_count[w], bins_used = max(bins_used, wave_last[w]);
        for (int b = tid; b < (int)bins_used; b += kPartThreads) a.bins[i * kSampleBins + b] = bins[kSampleBins - 1 - b];
        write_part(record, a.part[i], top, place, bins_used, count);
    }
}

// ---- gather ------------------------------------------------------------------------------------------------------------

// A part's entries down to the border's bin (or of that bin), in their order, to the row's list where the part found room: the counts
// of 64 vectors each are scanned 16 bits apiece.  Parts whose own bins say that there are none end before they read.  (The entries put
// together in LDS first and stored 64 at a time: 64 x 151,936 21 us for 16, flat rows 55 for 35, as that takes a barrier and registers.)
template <typename DT>
__global__ __launch_bounds__(kPartThreads, DT::kBytes == 4 ? 4 : 5) void sample_gather_kernel(SampleArgs a, int64_t row0, int64_t rows)
{
    using Entries = PartEntries<DT>;
    constexpr int EPV = Entries::EPV, kVectors = Entries::kVectors;
    __shared__ uint32_t wave_count[kPartWaves], start;
    __shared__ double wave_mass[kPartWaves];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    for (int64_t i = blockIdx.x; i < rows * a.parts; i += gridDim.x) {
        const int64_t r = i / a.parts, t = row0 + r;
        SampleRow &row = a.row[r];
        const SamplePart part = a.part[i];
        // (asked for before it is known whether they are needed, or there)
        constexpr int kEach = kSampleBins / kPartThreads;
        uint64_t bins[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) bins[j] = a.bins[i * kSampleBins + j * kPartThreads + tid];
        if (row.mode != kSampleFew && row.mode != kSampleBin) continue;
        SampleSegment out;
        out.above = 0.0, out.start = out.listed = 0;
        // the part's own bins that are looked for: up to `last`, of many only that one
        const int shift = part.max > -kInf ? row.place - part.place : 0;  // part's bin 0 is the row's bin `shift`
        const bool few = row.mode == kSampleFew, all = row.bin == kSampleAll;
        const int last = all ? kSampleAll : row.bin - shift;
        if (part.max > -kInf && last >= 0) {
            uint32_t n = 0;
            double above = 0.0;
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const int b = j * kPartThreads + tid;
                if (b < (int)part.bins) {
                    if (few ? b <= last : b == last) n += (uint32_t)(bins[j] >> kWeightBits);
                    if (!few && b < last) above += (double)(bins[j] & kWeightMask) * down_by((b + shift) << row.coarse);
                }
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
                if (tid == 0) start = atomicAdd(&row.cursor, n);  // (while the entries are on their way)
                const int64_t begin = (i - r * a.parts) * kSamplePart;
                Entries z;
                z.load(reinterpret_cast<const char *>(a.z) + (t * a.ld + begin) * DT::kBytes, (int)min(a.V - begin, (int64_t)kSamplePart));
                const float from = row.from, to = row.to;
                uint32_t taken = 0;  // a bit an entry
                z.each([&](float x, int k) { taken |= (x >= from && x <= to ? 1u : 0u) << k; });
                // how many of each 64 vectors are before a lane's, 16 bits each
                uint32_t pos[(kVectors + 1) / 2], sum[(kVectors + 1) / 2], in_wave = 0;
#pragma unroll
                for (int w = 0; w < (kVectors + 1) / 2; ++w) {
                    uint32_t own = 0;
#pragma unroll
                    for (int h = 0; h < 2; ++h) own |= (uint32_t)__popc(taken >> ((2 * w + h) * EPV) & ((1u << EPV) - 1)) << (16 * h);
                    const uint32_t scan = wave_scan(own);
                    pos[w] = scan - own;
                    sum[w] = last_lane(scan);
                    in_wave += (sum[w] & 0xFFFFu) + (sum[w] >> 16);
                }
                __syncthreads();  // (wave_count has been read)
                if (lane == 0) wave_count[wave] = in_wave;
                __syncthreads();
                out.start = start;
                uint32_t base = start;
#pragma unroll
                for (int w = 0; w < kPartWaves; ++w) base += w < wave ? wave_count[w] : 0;
                uint2 *list = a.list + r * kSampleListed;
#pragma unroll
                for (int v = 0; v < kVectors; ++v) {
                    uint32_t at = base + (pos[v / 2] >> (16 * (v & 1)) & 0xFFFFu);
                    float x[EPV];
                    unpack<DT>(z.raw[v], x);
#pragma unroll
                    for (int k = 0; k < EPV; ++k)
                        if (taken >> (v * EPV + k) & 1u) {
                            if (at < kSampleListed)
                                list[at] = make_uint2(__float_as_uint(x[k]), (uint32_t)(begin + Entries::first() + v * kWave * EPV + k));
                            ++at;
                        }
                    base += sum[v / 2] >> (16 * (v & 1)) & 0xFFFFu;
                }
            }
        }
        if (tid == 0) {
            SampleSegment &to = a.segment[i];
            to.above = out.above, to.start = out.start, to.listed = out.listed;
        }
    }
}

// ---- rows and finish -------------------------------------------------------------------------------------------------

// What the waves of a workgroup tell one another.  Two sets of places in turn: between a wave's writes to one and the reads of
// it two turns before lies the barrier of the turn between.
struct Turn {
    uint64_t whole[kWaves];
    double sum[kWaves], other[kWaves];
    uint32_t count[kWaves], more[kWaves];
    float top[kWaves], low[kWaves];
};
struct Scans {
    Turn turn[2];
    double table[32], told[2];
    float told_top;
    uint64_t found_mass;
    uint32_t found_digit, found_count, gathered;
    Border found;
    int64_t token;
    float token_logit, entries[16];
};
struct Shared : Scans {
    union {
        struct {  // entries of the row by bits of their keys
            uint64_t mass[kBins];
            uint32_t count[kBins];
        } key;
        struct {
            union {
                float value[kSampleListed];
                struct {
                    float few_values[kSampleFewest];
                    int32_t index[kSampleFewest];  // (only where they are few)
                };
            };
            uint64_t bin_mass[kThreads];
            uint32_t bin_count[kThreads];
        } list;
    };
    uint64_t block_mass[kSampleBlocks];
    uint32_t block_count[kSampleBlocks];
};
static_assert(kSampleListed == 2 * kSampleFewest, "few values leave room for their indices");
static_assert(kSampleBlocks == kThreads && kSampleBins == kThreads, "a block and a bin a thread");

// Sum over the waves before a thread's own, and over all: of N / 64 waves' totals, which the lanes of each wave add up.
template <int N, typename T>
__device__ __forceinline__ T before_wave(const T *totals, T &total)
{
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const T v = lane < N / kWave ? totals[lane] : T(0), upto = wave_scan(v);
    total = last_lane(upto);
    // (scan less own would round sums of floats)
    const T before = from_lanes<0x138, 0xF>(upto);  // of the lane before
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, before), wave));
    } else {
        const uint64_t u = __builtin_bit_cast(uint64_t, before);
        return __builtin_bit_cast(T, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), wave) << 32 |
                                         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, wave));
    }
}

// Sums over the threads before and up to each, and over all; N threads, TURN 0 and 1 in turn.
template <int N, int TURN>
__device__ __forceinline__ void block_scan(Scans &sh, uint64_t &mass, uint32_t &count, uint64_t &mass_total, uint32_t &count_total)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    mass = wave_scan(mass);
    count = wave_scan(count);
    if (lane == kWave - 1) sh.turn[TURN].whole[wave] = mass, sh.turn[TURN].count[wave] = count;
    __syncthreads();
    mass += before_wave<N>(sh.turn[TURN].whole, mass_total);
    count += before_wave<N>(sh.turn[TURN].count, count_total);
}
template <int N, int TURN>
__device__ __forceinline__ void block_scan(Scans &sh, uint32_t &count, uint32_t &count_total)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    count = wave_scan(count);
    if (lane == kWave - 1) sh.turn[TURN].count[wave] = count;
    __syncthreads();
    count += before_wave<N>(sh.turn[TURN].count, count_total);
}
// `other` and `more` are only summed
template <int N, int TURN>
__device__ __forceinline__ void block_scan(Scans &sh, double &sum, double &total, double &other, uint32_t &count, uint32_t &count_total, uint32_t &more)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    sum = wave_scan(sum);
    count = wave_scan(count);
    other = wave_sum(other);
    more = wave_sum(more);
    Turn &t = sh.turn[TURN];
    if (lane == kWave - 1) t.sum[wave] = sum, t.count[wave] = count, t.other[wave] = other, t.more[wave] = more;
    __syncthreads();
    double all_other;
    uint32_t all_more;
    sum += before_wave<N>(t.sum, total);
    count += before_wave<N>(t.count, count_total);
    (void)before_wave<N>(t.other, all_other);
    (void)before_wave<N>(t.more, all_more);
    other = all_other, more = all_more;
}
template <int N, int TURN>
__device__ __forceinline__ void block_scan(Scans &sh, double &sum, double &total)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    sum = wave_scan(sum);
    if (lane == kWave - 1) sh.turn[TURN].sum[wave] = sum;
    __syncthreads();
    sum += before_wave<N>(sh.turn[TURN].sum, total);
}
// the first thread for which `here` holds, or else the last for which `other` does (-1: none)
template <int N, int TURN>
__device__ __forceinline__ int block_first(Scans &sh, bool here, bool other)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const uint64_t a = __ballot(here), b = __ballot(other);
    // (a wave's first and last thread, 0 for none)
    if (lane == 0) {
        sh.turn[TURN].count[wave] = a ? wave * kWave + __builtin_ctzll(a) + 1 : 0;
        sh.turn[TURN].more[wave] = b ? wave * kWave + 64 - __builtin_clzll(b) : 0;
    }
    __syncthreads();
    const uint32_t first = lane < N / kWave ? sh.turn[TURN].count[lane] : 0, last = lane < N / kWave ? sh.turn[TURN].more[lane] : 0;
    const uint64_t firsts = __ballot(first != 0), lasts = __ballot(last != 0);
    if (firsts) return __builtin_amdgcn_readlane((int)first, __builtin_ctzll(firsts)) - 1;
    return lasts ? __builtin_amdgcn_readlane((int)last, 63 - __builtin_clzll(lasts)) - 1 : -1;
}
// the largest and the smallest over the workgroup
template <int N, int TURN>
__device__ __forceinline__ void block_range(Scans &sh, float &high, float &low)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    high = wave_max(high), low = wave_max(-low);
    if (lane == 0) sh.turn[TURN].top[wave] = high, sh.turn[TURN].low[wave] = low;
    __syncthreads();
    high = wave_max(lane < N / kWave ? sh.turn[TURN].top[lane] : -kInf);
    low = -wave_max(lane < N / kWave ? sh.turn[TURN].low[lane] : -kInf);
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
    __device__ __forceinline__ uint4 load_raw(int64_t e) const  // -inf behind the row's end
    {
        if (e + kEpv <= V) return row_load<true, true>(p + e * DT::kBytes);
        uint4 v = neg_inf_vec<DT>();
        if (e < V) {
            float f[kEpv];
#pragma unroll
            for (int k = 0; k < kEpv; ++k) f[k] = e + k < V ? load_elem<DT>(p, e + k) : -kInf;
            v = pack<DT>(f);
        }
        return v;
    }
    __device__ __forceinline__ void load(int64_t e, float *f) const { unpack<DT>(load_raw(e), f); }
    // f(values, first entry, block) of every 64 vectors of the row, a wavefront each, its loads kAhead together
    template <typename F>
    __device__ __forceinline__ void each(F f) const
    {
        constexpr int kAhead = 4;
        for (int s = 0; s < steps; ++s)
#pragma unroll 1
            for (int b = threadIdx.x / kWave; b < blocks; b += kWaves * kAhead) {
                uint4 raw[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) raw[i] = load_raw(first(b + i * kWaves, s));
#pragma unroll 1
                for (int i = 0; i < kAhead; ++i) {
                    float v[kEpv];
                    unpack<DT>(raw[0], v);
#pragma unroll
                    for (int j = 1; j < kAhead; ++j) raw[j - 1] = raw[j];
                    if (b + i * kWaves < blocks) f(v, first(b + i * kWaves, s), b + i * kWaves);
                }
            }
    }
};

// What is written for the drawn token, which its thread has left in sh; sums are in units of 2^-shift of the largest weight.
__device__ __forceinline__ void tell(const SampleArgs &a, Scans &sh, int64_t t, float top, float tau, int shift, double kept_mass, double full_mass, uint32_t kept)
{
    __syncthreads();
    if (threadIdx.x >= 2) return;
    const double x = ((double)sh.token_logit - (double)top) / (double)tau, unit = shift * 0.69314718055994530942;
    // (a thread each: the logarithm is there once)
    float *to = threadIdx.x ? a.logp_full : a.logp;
    if (to) to[t] = (float)fmin(x - (log(threadIdx.x ? full_mass : kept_mass) - unit), 0.0);  // (sums' rounding: a few 2^-52 too little)
    if (threadIdx.x == 0) {
        a.token[t] = (int32_t)sh.token;
        if (a.kept) a.kept[t] = (int32_t)kept;
    }
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
#pragma unroll 1
        for (int i = threadIdx.x; i < kBins; i += kThreads) sh.key.mass[i] = 0, sh.key.count[i] = 0;
        __syncthreads();
        const uint32_t mask = (1u << bits) - 1;
        row.each([&](const float *v, int64_t, int) {
            // (64 vectors of one value are added by one lane: additions to one place wait for one another)
            const float one = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v[0])));
            bool same = true;
#pragma unroll
            for (int k = 0; k < EPV; ++k) same &= v[k] == one;
            const uint32_t times = __all(same) ? kWave * EPV : 1;
#pragma unroll
            for (int k = 0; k < EPV; ++k) {
                const uint32_t key = key_of(v[k]);
                if (times > 1 && (k > 0 || threadIdx.x % kWave != 0)) continue;
                if (key > kKeyOfNegInf && (bits + shift == 32 || key >> (shift + bits) == prefix)) {
                    const uint32_t d = key >> shift & mask;
                    atomicAdd(&sh.key.count[d], times);
                    atomicAdd(reinterpret_cast<unsigned long long *>(&sh.key.mass[d]), (unsigned long long)weigh.whole(v[k]) * times);
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
        __syncthreads();
        block_scan<kThreads, 0>(sh, mi, ci, mass_total, count_total);
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
        uint32_t upto = own, all_equal;
        block_scan<kThreads, 1>(sh, upto, all_equal);
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
                const uint32_t all = last_lane(scan);
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
        if (!policy.by_k() && !policy.by_p()) return border;
        histogram(0, 20, 12);
        uint64_t mass = 0, total;
        uint32_t count = 0, finite;
        find<true>(1, mass, count, total, finite);
        if (policy.by_k() && policy.k < finite) {
            border = select<false>((uint64_t)policy.k, total);
            if (policy.by_p()) histogram(0, 20, 12);
        }
        if (policy.by_p()) {
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
            const uint64_t sum = wave_sum((uint64_t)in_block);
            if (lane == 0) sh.block_mass[b] = sum;
        }
        uint64_t full_total, total;
        uint32_t kept, none, zero = 0;
        block_scan<kThreads, 0>(sh, full, mine, full_total, kept);
        const uint64_t own = sh.block_mass[tid];  // (written before the scan's barrier)
        uint64_t mass = own;
        block_scan<kThreads, 1>(sh, mass, zero, total, none);
        // the block, then the entry, in whose part of the sum the number falls
        const uint64_t target = (uint64_t)((double)policy.u * (double)total);
        if (mass > target && mass - own <= target) sh.found_digit = tid, sh.found_mass = target - (mass - own);
        __syncthreads();
        if (wave == 0) {
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
                const uint64_t upto = wave_scan(sum);
                if (upto > left && upto - sum <= left) {
                    uint64_t at = upto - sum;
                    bool done = false;
#pragma unroll
                    for (int i = 0; i < EPV; ++i) {
                        at += border.keeps(v[i], (int32_t)(e + i)) ? weigh.whole(v[i]) : 0;
                        if (!done && at > left) sh.token = e + i, sh.token_logit = v[i], done = true;
                    }
                }
                if (__any(upto > left)) break;
                left -= last_lane(upto);
            }
        }
        tell(a, sh, t, top, policy.tau, a.shift, (double)total, (double)full_total, kept);
    }
};

template <int N>
__device__ __forceinline__ void tell_none(const SampleArgs &a, int64_t t, bool bad)
{
    if (a.allowed)
        for (int64_t w = threadIdx.x; w < (a.V + 31) / 32; w += N) a.allowed[t * a.allowed_ld + w] = 0;
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

// Of so many entries from `begin` on, kEach a thread, the one in whose part of the kept sum the number falls; `within`: what of it lies there, in
// units of the weight of weigh's maximum times what its table is scaled by.  At least one of them is kept and has a weight beside that
// maximum (callers choose by masses that are zero elsewhere), so there is such a thread.  Turns 0 and 1, in this order.
template <int N, int kEach, typename DT>
__device__ __forceinline__ void draw(Scans &sh, const Row<DT> &row, const Weigh &weigh, int64_t begin, int entries, double within, Border border)
{
    constexpr int EPV = DT::kPerVec;
    const int tid = threadIdx.x;
    const int64_t e = begin + tid * kEach;
    const bool active = tid * kEach < entries;
    uint4 raw[kEach / EPV];
#pragma unroll
    for (int k = 0; k < kEach / EPV; ++k) raw[k] = active ? row.load_raw(e + k * EPV) : neg_inf_vec<DT>();
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < kEach / EPV; ++k) {
        float v[EPV];
        unpack<DT>(raw[k], v);
#pragma unroll
        for (int j = 0; j < EPV; ++j) sum += border.keeps(v[j], (int32_t)(e + k * EPV + j)) ? weigh(v[j]) : 0.0;
        asm volatile("" : "+v"(sum));
    }
    double scan = sum, all;
    block_scan<N, 0>(sh, scan, all);
    const int thread = block_first<N, 1>(sh, scan > within && sum > 0.0, sum > 0.0);
    if (tid == thread) {
#pragma unroll
        for (int k = 0; k < kEach / EPV; ++k) {
            float v[EPV];
            unpack<DT>(raw[k], v);
#pragma unroll
            for (int j = 0; j < EPV; ++j) sh.entries[k * EPV + j] = v[j];
        }
        sh.told[1] = scan - sum;
    }
    __syncthreads();
    if (tid < kWave) {
        // its entries, a lane each
        const float v = tid < kEach ? sh.entries[tid] : -kInf;
        const int64_t at = begin + (int64_t)thread * kEach + tid;
        const double w = tid < kEach && border.keeps(v, (int32_t)at) ? weigh(v) : 0.0, upto = sh.told[1] + wave_scan(w);
        const uint64_t here = __ballot(w > 0.0 && upto > within), some = __ballot(w > 0.0);
        if (tid == (here ? __builtin_ctzll(here) : 63 - __builtin_clzll(some | 1))) sh.token = at, sh.token_logit = v;
    }
}

// What all parts say together: the maximum, NaN where there is no policy, and whether one is off the grid.  The thread's own part is
// left in `mine`.  Turn 0.
template <int N>
__device__ __forceinline__ float top_of(const SampleArgs &a, Scans &sh, const SamplePart *part, SamplePart &mine, bool &far)
{
    float top = -kInf;
    bool bad = false, off = false;
    mine = {};
    mine.max = -kInf;
    for (int q = threadIdx.x; q < a.parts; q += N) {
        mine = part[q];
        top = fmaxf(top, mine.max), bad |= mine.max != mine.max, off |= mine.max > -kInf && mine.place == kSampleFar;
    }
    float worst = bad ? 0.0f : off ? 1.0f : 2.0f;
    block_range<N, 0>(sh, top, worst);
    far = worst == 1.0f;
    return worst == 0.0f ? __builtin_nanf("") : top;
}

// An uncut row: the part, a quarter of it, the entry, in whose part of the sum the number falls.  Turns 1, 0, ...
template <int N, typename DT>
__device__ __forceinline__ void draw_uncut(const SampleArgs &a, Scans &sh, const Policy &policy, const SamplePart &mine, int64_t t, float top)
{
    const int tid = threadIdx.x;
    const double unit = kUnit / (double)policy.tau;
    const Weigh weigh{(double)top, unit, sh.table};
    // what the part's weights are relative to, in units of 2^-shift of the row's largest, and of its own
    const double scale = ldexp(1.0, a.shift);
    const bool some = mine.max > -kInf, wide = is_wide(mine.max, unit);
    const double factor = !some ? 0.0 : wide ? weigh(mine.max) : scale * exp2((double)top * unit * -0.03125);
    const double own = (mine.mass[0] + mine.mass[1] + mine.mass[2] + mine.mass[3]) * factor;
    double upto = own, full, none = 0.0;
    uint32_t finite = mine.count, kept, more = 0;
    block_scan<N, 1>(sh, upto, full, none, finite, kept, more);
    const double target = (double)number_of(policy) * full;
    const int chosen = block_first<N, 0>(sh, upto > target && own > 0.0, own > 0.0);
    if (tid == chosen) {
        double within = fmax(target - (upto - own), 0.0) / factor;
        const double m0 = mine.mass[0], m1 = mine.mass[1], m2 = mine.mass[2], m3 = mine.mass[3];
        const int last = m3 > 0.0 ? 3 : m2 > 0.0 ? 2 : m1 > 0.0 ? 1 : 0;
        int quarter = 0;
        if (last > 0 && !(m0 > within)) within -= m0, quarter = 1;
        if (quarter == 1 && last > 1 && !(m1 > within)) within -= m1, quarter = 2;
        if (quarter == 2 && last > 2 && !(m2 > within)) within -= m2, quarter = 3;
        sh.told[0] = within * (wide ? 1.0 : exp2((double)mine.max * unit * -0.03125)) * scale;
        sh.told_top = mine.max;
        sh.found_digit = chosen * kPartWaves + quarter;
    }
    __syncthreads();
    const Weigh here{(double)sh.told_top, unit, sh.table};
    const Row<DT> row{reinterpret_cast<const char *>(a.z) + t * a.ld * DT::kBytes, a.V, a.steps, a.blocks};
    constexpr int kQuarter = kSamplePart / kPartWaves;
    draw<N, 8>(sh, row, here, (int64_t)sh.found_digit * kQuarter, kQuarter, sh.told[0], Border{kKeyOfNegInf, -1});
    tell(a, sh, t, top, policy.tau, a.shift, full, full, kept);
}

// Rows that the host knows to be uncut.
template <typename DT>
__global__ __launch_bounds__(kPartThreads, 4) void sample_uncut_kernel(SampleArgs a, int64_t row0, int64_t rows)
{
    __shared__ Scans sh;
    if (threadIdx.x < 32) sh.table[threadIdx.x] = ldexp(kTable[threadIdx.x], a.shift);
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        SamplePart mine;
        bool far;
        __syncthreads();  // (the row before this one is done with everything)
        const float top = top_of<kPartThreads>(a, sh, a.part + r * a.parts, mine, far);
        const Policy policy(a, row0 + r);
        if (policy.bad() || !(top > -kInf)) tell_none<kPartThreads>(a, row0 + r, policy.bad() || top != top);
        else draw_uncut<kPartThreads, DT>(a, sh, policy, mine, row0 + r, top);
    }
}

// ---- rows --------------------------------------------------------------------------------------------------------------

// A row: its parts' bins added up, a bin a thread, the borders' bin, and how the row goes on: its entries down to there listed (few), that
// bin's alone, or in passes.  Uncut rows among cut ones get their token here.
template <typename DT>
__global__ __launch_bounds__(kThreads, 4) void sample_rows_kernel(SampleArgs a, int64_t row0, int64_t rows)
{
    __shared__ Scans sh;
    __shared__ int part_place[kThreads];
    __shared__ uint32_t part_bins[kThreads];
    const int tid = threadIdx.x;
    if (tid < 32) sh.table[tid] = ldexp(kTable[tid], a.shift);
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const int64_t t = row0 + r;
        SamplePart mine;
        bool far;
        __syncthreads();  // (the row before this one is done with everything)
        const Policy policy(a, t);
        const float top = top_of<kThreads>(a, sh, a.part + r * a.parts, mine, far);
        const bool each_part = a.parts <= kThreads;
        const double unit = kUnit / (double)policy.tau;
        SampleRow out;
        out.full = out.above = out.share = 0.0, out.rank = 0, out.top = top;
        out.mode = kSamplePasses, out.by_k = out.place = out.bin = 0, out.count = 0, out.from = out.to = 0.0f;
        if (policy.bad() || !(top > -kInf)) {
            tell_none<kThreads>(a, t, policy.bad() || top != top);
            out.mode = kSampleDone;
        } else if (!policy.cut() && each_part) {
            draw_uncut<kThreads, DT>(a, sh, policy, mine, t, top);
            out.mode = kSampleDrawn;
        } else if (policy.cut() && each_part && !far) {
            // ---- all parts' bins on the row's grid, a bin a thread
            const int coarse = policy.coarse();
            const double grid = unit * (coarse ? 0.125 : 0.5), step = kPlace * (double)policy.tau * (coarse ? 4.0 : 1.0);
            const float lowest = lowest_of(policy.tau);
            out.place = place_of(top, grid, lowest);
            const bool some = mine.max > -kInf;
            part_place[tid] = some ? mine.place : 0, part_bins[tid] = some ? mine.bins : 0;
            const int64_t apart = some ? (int64_t)out.place - mine.place : 0;
            double mass = some && apart < 16000 >> coarse ? mine.mass[0] + mine.mass[1] + mine.mass[2] + mine.mass[3] : 0.0;
            if (mass > 0.0) mass *= down_by((int)apart << coarse) * kOne;
            __syncthreads();
            uint64_t sum = 0;
            uint32_t own_count = 0;
            const uint64_t *bins = a.bins + r * a.parts * kSampleBins;
            constexpr int kTogether = 8;
#pragma unroll 1
            for (int first = 0; first < a.parts; first += kTogether) {
                uint64_t v[kTogether];
#pragma unroll
                for (int j = 0; j < kTogether; ++j) {
                    // (what is not there is read all the same, from within the array, and left out below)
                    const int q = min(first + j, a.parts - 1);
                    const uint32_t b = (uint32_t)tid - ((uint32_t)out.place - (uint32_t)part_place[q]);
                    v[j] = bins[q * kSampleBins + min(b, (uint32_t)kSampleBins - 1)];
                }
#pragma unroll
                for (int j = 0; j < kTogether; ++j) {
                    const int q = min(first + j, a.parts - 1);
                    const uint32_t b = (uint32_t)tid - ((uint32_t)out.place - (uint32_t)part_place[q]);
                    const bool there = first + j < a.parts && b < part_bins[q];
                    sum += there ? v[j] & kWeightMask : 0, own_count += there ? (uint32_t)(v[j] >> kWeightBits) : 0;
                }
            }
            // in units of the weight in the middle of bin 0, times 2^36
            const double own = (double)sum * down_by(tid << coarse);
            double upto = own, all;
            uint32_t count = own_count, binned, finite = mine.count;
            block_scan<kThreads, 1>(sh, upto, all, mass, count, binned, finite);
            out.full = mass;
            // ---- the bin of the tightest border; several may share it
            const bool by_k = policy.by_k() && policy.k < (int64_t)finite;
            const double need = (double)fmaxf(policy.p, 0.0f) * out.full;
            bool lost = false;
            int bin = kSampleAll, bin_p = -1;
            if (by_k || policy.by_p()) {
                bin = block_first<kThreads, 0>(sh, own_count > 0 && (by_k ? (int64_t)count >= policy.k : upto >= need), false);
                if (bin < 0) bin = kSampleAll, lost = true;
                else if (!by_k) bin_p = bin;
            }
            const int bin_k = by_k ? bin : -1;
            // (top_p is a share of what top_k leaves, so with both all of that is needed)
            if (policy.by_min() && !(by_k && policy.by_p())) {
                const int64_t b = (int64_t)out.place - place_of(least_of(policy, top), grid, lowest);
                if (b < kSampleBins && b < bin) bin = (int)b, lost = false;
            }
            // how many there are down to it, and in it
            if (tid == 0) sh.found_count = finite, sh.found_digit = 0, sh.told[0] = 0.0;
            __syncthreads();
            if (tid == bin) sh.found_count = count, sh.found_digit = own_count, sh.told[0] = upto - own;
            __syncthreads();
            const uint32_t down_to = sh.found_count, in_bin = sh.found_digit;
            out.bin = bin;
            out.above = sh.told[0];
            out.count = down_to - in_bin;
            out.share = bin_p == bin ? need : -1.0;
            out.rank = bin_k == bin && by_k ? policy.k - out.count : -1;
            out.by_k = by_k;
            if (down_to <= kSampleFewest) out.mode = kSampleFew;
            else if (!lost && bin != kSampleAll && in_bin <= kSampleListed && !(by_k && policy.by_p())) out.mode = kSampleBin;
            if (out.mode != kSamplePasses) {
                out.from = bin == kSampleAll ? -3.402823466e38f : first_at(out.place - bin, grid, step, lowest);
                out.to = out.mode == kSampleFew ? kInf : nextafterf(first_at(out.place - bin + 1, grid, step, lowest), -kInf);
            }
        }
        // (field by field: a whole struct's copy takes its padding along, through a private array that ends up in LDS by a thread
        // number from the dispatch packet in host memory, 4 to 14 us at the kernel's beginning)
        if (tid == 0) {
            SampleRow &to = a.row[r];
            to.full = out.full, to.above = out.above, to.share = out.share, to.rank = out.rank, to.top = out.top;
            to.mode = out.mode, to.by_k = out.by_k, to.place = out.place, to.bin = out.bin, to.count = out.count, to.cursor = 0;
            to.from = out.from, to.to = out.to, to.coarse = policy.coarse();
            to.key = kKeyOfNegInf, to.last = -1;  // (all above -inf; of cut rows finish says it)
        }
    }
}

// ---- finish ------------------------------------------------------------------------------------------------------------

// The gathered entries; positions are in the order of the indices.  The last entry kept, by its logit and its position.
struct Last {
    float value;
    uint32_t position;
    __device__ __forceinline__ bool keeps(float v, uint32_t q) const { return v > value || (v == value && q <= position); }
};
__device__ __forceinline__ Last tighter(Last a, Last b)
{
    if (a.value != b.value) return a.value > b.value ? a : b;
    return Last{a.value, min(a.position, b.position)};
}

// Of n entries between low and high, the last of those that make `target`, whole numbers: a count, or a mass.  mass: up to it.
// Bins, then the bins of one bin, until few enough are left to compare each with all others, or all left are equal.
__device__ __forceinline__ Last last_of(Shared &sh, const Weigh &weigh, uint32_t n, float high, float low, bool by_mass, uint64_t target, uint64_t &mass)
{
    const int tid = threadIdx.x;
    uint32_t m = n, count_before = 0;
    uint64_t mass_before = 0;
#pragma unroll 1
    while (m > kDirect && low < high) {
        const float scale = (float)(kThreads - 1) / (high - low);
        auto bin_of = [&](float v) {
            const int b = (int)fminf(fmaxf((high - v) * scale, 0.0f), (float)(kThreads - 1));
            return v == low ? kThreads - 1 : v == high ? 0 : b;  // (apart whatever the scale is)
        };
        __syncthreads();
        sh.list.bin_mass[tid] = 0, sh.list.bin_count[tid] = 0;
        __syncthreads();
#pragma unroll 1
        for (uint32_t i = tid; i < n; i += kThreads) {
            const float v = sh.list.value[i];
            if (v >= low && v <= high) {
                const int b = bin_of(v);
                atomicAdd(&sh.list.bin_count[b], 1u);
                atomicAdd(reinterpret_cast<unsigned long long *>(&sh.list.bin_mass[b]), (unsigned long long)weigh.whole(v));
            }
        }
        __syncthreads();
        const uint64_t own = sh.list.bin_mass[tid];
        const uint32_t own_count = sh.list.bin_count[tid];
        uint64_t upto = own, all;
        uint32_t count = own_count, all_count;
        block_scan<kThreads, 0>(sh, upto, count, all, all_count);
        if (by_mass) target = min(target, mass_before + all);  // (rounding may ask for more than there is)
        upto += mass_before, count += count_before;
        if (by_mass ? upto >= target && upto - own < target : count >= target && count - own_count < target)
            sh.found_digit = tid, sh.found_mass = upto - own, sh.found_count = count - own_count;
        __syncthreads();
        const int bin = (int)sh.found_digit;
        mass_before = sh.found_mass, count_before = sh.found_count;
        m = sh.list.bin_count[bin];
        float h = -kInf, l = kInf;
#pragma unroll 1
        for (uint32_t i = tid; i < n; i += kThreads) {
            const float v = sh.list.value[i];
            if (v >= low && v <= high && bin_of(v) == bin) h = fmaxf(h, v), l = fminf(l, v);
        }
        block_range<kThreads, 1>(sh, h, l);
        high = h, low = l;
    }
    __syncthreads();
    if (m <= kDirect) {
        uint32_t *at = sh.block_count;
        uint64_t *weight = sh.block_mass;
        float *value = reinterpret_cast<float *>(sh.list.bin_count);
        if (tid == 0) sh.gathered = 0;
        at[tid] = 0, weight[tid] = 0, value[tid] = -kInf;
        __syncthreads();
#pragma unroll 1
        for (uint32_t i = tid; i < n; i += kThreads) {
            const float v = sh.list.value[i];
            if (v >= low && v <= high) {
                const uint32_t to = atomicAdd(&sh.gathered, 1u);
                at[to] = i, value[to] = v;
                weight[to] = weigh.whole(v);
            }
        }
        __syncthreads();
        if ((uint32_t)tid < m) {
            const uint32_t mine = at[tid];
            const float v = value[tid];
            uint64_t ahead = mass_before, all = mass_before;
            uint32_t before = count_before;
#pragma unroll 1
            for (uint32_t q = 0; q < m; q += 8)
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) {  // (behind the m-th there is nothing, at -inf)
                    const float o = value[q + j];
                    const uint64_t w = weight[q + j];
                    const uint32_t first = (uint32_t)(o > v) | ((uint32_t)(o == v) & (uint32_t)(at[q + j] < mine));
                    ahead += w & (0ull - first);
                    all += w;
                    before += first;
                }
            if (by_mass) target = min(target, all);
            if (by_mass ? ahead < target && ahead + weight[tid] >= target : before + 1 == target)
                sh.found = Border{__float_as_uint(v), (int32_t)mine}, sh.found_mass = ahead + weight[tid];
        }
    } else {
        // all the m left are equal: the c-th of them
        const uint64_t each = weigh.whole(high), left = target - (by_mass ? mass_before : count_before);
        const uint32_t c = by_mass ? (uint32_t)min((left + each - 1) / (each ? each : 1), (uint64_t)m) : (uint32_t)left;
        const uint32_t run = (n + kThreads - 1) / kThreads;
        uint32_t own = 0, all;
        for (uint32_t i = tid * run; i < min(n, (tid + 1) * run); ++i) own += sh.list.value[i] == high ? 1u : 0u;
        uint32_t upto = own;
        block_scan<kThreads, 0>(sh, upto, all);
        if (upto >= c && upto - own < c) {
            uint32_t k = upto - own;
            for (uint32_t i = tid * run; i < min(n, (tid + 1) * run); ++i)
                if (sh.list.value[i] == high && ++k == c) sh.found = Border{__float_as_uint(high), (int32_t)i}, sh.found_mass = mass_before + c * each;
        }
    }
    __syncthreads();
    mass = sh.found_mass;
    return Last{__uint_as_float(sh.found.key), (uint32_t)sh.found.last};
}

// Rows that the bins do not settle, as often as their cuts ask.
template <typename DT>
__global__ __launch_bounds__(kThreads, 4) void sample_passes_kernel(SampleArgs a, int64_t row0, int64_t rows)
{
    __shared__ Shared sh;
#pragma unroll 1
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const int64_t t = row0 + r;
        if (a.row[r].mode != kSamplePasses) continue;
        __syncthreads();
        if (threadIdx.x < 32) sh.table[threadIdx.x] = ldexp(kTable[threadIdx.x], a.shift);
        __syncthreads();  // (the table is there; the row before this one is done with everything)
        const float top = a.row[r].top;
        Policy policy(a, t);
        policy.u = number_of(policy);
        const Weigh weigh{(double)top, kUnit / (double)policy.tau, sh.table};
        Passes<DT> passes{a, sh, Row<DT>{reinterpret_cast<const char *>(a.z) + t * a.ld * DT::kBytes, a.V, a.steps, a.blocks}, weigh};
        Border border{kKeyOfNegInf, -1};
        if (policy.by_min()) border = Border{key_of(fmaxf(least_of(policy, top), -3.402823466e38f)), kAnyIndex};
        passes.finish(policy, tighter(border, passes.cut(policy)), t, top);
    }
}

// A row's border among its listed entries, and its token.  (With the rows that go in passes taken here too, for a launch less, their
// registers are everyone's: 64 x 151,936 30 us for the 20 + 4 of both kernels.)
template <typename DT>
__global__ __launch_bounds__(kThreads, 4) void sample_finish_kernel(SampleArgs a, int64_t row0, int64_t rows)
{
    __shared__ Shared sh;
    const int tid = threadIdx.x, shift = max(a.shift, kSampleListShift);
    if (tid < 32) sh.table[tid] = ldexp(kTable[tid], shift);
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const int64_t t = row0 + r;
        // (asked for before it is known whether they are needed, or there)
        const SampleRow &row = a.row[r];
        const SampleSegment segment_read = a.segment[r * a.parts + min(tid, a.parts - 1)];
        Policy policy(a, t);
        if (row.mode != kSampleFew && row.mode != kSampleBin) continue;
        __syncthreads();  // (the table is there; the row before this one is done with everything)
        policy.u = number_of(policy);
        const float top = row.top;
        const double unit = kUnit / (double)policy.tau;
        const Weigh weigh{(double)top, unit, sh.table};
        const Row<DT> data{reinterpret_cast<const char *>(a.z) + t * a.ld * DT::kBytes, a.V, a.steps, a.blocks};
        const float least = policy.by_min() ? fmaxf(least_of(policy, top), -3.402823466e38f) : -3.402823466e38f;
        // what one unit of the bins' sums (2^-36 of the middle of bin 0) is in units of 2^-shift of the largest weight
        const double to_whole = ldexp(exp2(fma(-(double)top, unit * 0.5, (double)row.place * (double)(1 << row.coarse)) * 0.0625), shift - 36);
        const double full = row.full * to_whole;
        const bool few = row.mode == kSampleFew;
        // ---- the gathered entries, from the order in which the parts found room to the parts' own
        SampleSegment segment = segment_read;
        if (tid >= a.parts) segment.above = 0.0, segment.start = segment.listed = 0;
        uint32_t place = segment.listed, n;  // where this thread's part's begin; entries
        block_scan<kThreads, 0>(sh, place, n);
        place -= segment.listed;
        sh.block_count[tid] = place - segment.start;
        __syncthreads();
        float high = -kInf, low = kInf;
        const uint2 *list = a.list + r * kSampleListed;
        constexpr int kTogether = 4;
#pragma unroll 1
        for (uint32_t first = tid; first < n; first += kThreads * kTogether) {
            uint2 v[kTogether];
#pragma unroll
            for (int j = 0; j < kTogether; ++j) v[j] = list[min(first + j * kThreads, n - 1)];  // (the last one again and again)
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {
                const uint32_t to = min(first + j * kThreads, n - 1) + sh.block_count[v[j].y / kSamplePart];
                const float x = __uint_as_float(v[j].x);
                sh.list.value[to] = x;
                if (few) sh.list.index[to] = (int32_t)v[j].y;
                high = fmaxf(high, x), low = fminf(low, x);
            }
        }
        block_range<kThreads, 1>(sh, high, low);
        // ---- the border among them
        Last border{least, 0xFFFFFFFFu};
        double total = full;  // of what top_p is a share of
        const int64_t k = few ? policy.k : row.rank;
        const bool by_k = few ? row.by_k && k <= (int64_t)n : k > 0;  // (min_p may end the list before the k-th; there is no top_p then)
        const bool by_p = few ? policy.by_p() : row.share >= 0.0;
#pragma unroll 1
        for (int which = 0; which < 2; ++which) {
            if (which == 0 ? !by_k : !by_p) continue;
            uint64_t target = (uint64_t)k, mass;
            if (which == 1) {
                const double need = ceil(few ? (double)fmaxf(policy.p, 0.0f) * total : (row.share - row.above) * to_whole);
                target = need < 1.0 ? 1 : (uint64_t)fmin(need, 0x1p62);  // (top_p may ask for far more than min_p has left in the list)
            }
            border = tighter(border, last_of(sh, weigh, n, high, low, which == 1, target, mass));
            if (which == 0) total = (double)mass;
        }
        __syncthreads();
        if (few) {
            // ---- the kept in the order of their indices, so many a thread
            const uint32_t run = (n + kThreads - 1) / kThreads;
            uint64_t sum = 0;
            uint32_t kept = 0;
#pragma unroll 1
            for (uint32_t q = tid * run; q < min(n, (tid + 1) * run); ++q)
                if (border.keeps(sh.list.value[q], q)) sum += weigh.whole(sh.list.value[q]), ++kept;
            uint64_t scan = sum, all;
            uint32_t kept_total;
            block_scan<kThreads, 1>(sh, scan, kept, all, kept_total);
            const uint64_t target = (uint64_t)((double)policy.u * (double)all);
            if (scan > target && scan - sum <= target) {
                uint64_t at = scan - sum;
#pragma unroll 1
                for (uint32_t q = tid * run; q < n; ++q) {
                    const float v = sh.list.value[q];
                    if (border.keeps(v, q)) at += weigh.whole(v);
                    if (at > target) {
                        sh.token = sh.list.index[q], sh.token_logit = v;
                        break;
                    }
                }
            }
            tell(a, sh, t, top, policy.tau, shift, (double)all, full, kept_total);
            if (a.allowed) {
                // bits of so many words at a time
                constexpr int kWords = 2 * kSampleBlocks;
                uint32_t *words = reinterpret_cast<uint32_t *>(sh.block_mass);
                const int64_t words_all = (a.V + 31) / 32;
#pragma unroll 1
                for (int64_t begin = 0; begin < words_all; begin += kWords) {
                    __syncthreads();
                    words[tid] = 0, words[tid + kThreads] = 0;
                    __syncthreads();
#pragma unroll 1
                    for (uint32_t q = tid; q < n; q += kThreads) {
                        const int32_t e = sh.list.index[q];
                        const int64_t w = (e >> 5) - begin;
                        if (w >= 0 && w < kWords && border.keeps(sh.list.value[q], q)) atomicOr(&words[w], 1u << (e & 31));
                    }
                    __syncthreads();
                    for (int64_t w = tid; w < kWords && begin + w < words_all; w += kThreads) a.allowed[t * a.allowed_ld + begin + w] = (int32_t)words[w];
                }
            }
            continue;
        }
        // ---- each part's kept: what is above the bin, and of the bin what is in its segment
        sh.block_count[tid] = place - segment.start, sh.block_mass[tid] = 0;
        // (the part that holds the border's position says its index)
        if (border.position - place < segment.listed) sh.found.last = (int32_t)list[segment.start + (border.position - place)].y;
        __syncthreads();
        const Border last{key_of(border.value), border.position == 0xFFFFFFFFu ? kAnyIndex : sh.found.last};
        uint32_t kept = 0;
#pragma unroll 1
        for (uint32_t first = tid; first < n; first += kThreads * kTogether) {
            uint2 v[kTogether];
#pragma unroll
            for (int j = 0; j < kTogether; ++j) v[j] = list[min(first + j * kThreads, n - 1)];
#pragma unroll 1
            for (int j = 0; j < kTogether && first + j * kThreads < n; ++j) {
                const uint2 u = v[0];
                v[0] = v[1], v[1] = v[2], v[2] = v[3];
                if (last.keeps(__uint_as_float(u.x), (int32_t)u.y)) {
                    atomicAdd(reinterpret_cast<unsigned long long *>(&sh.block_mass[u.y / kSamplePart]), (unsigned long long)weigh.whole(__uint_as_float(u.x)));
                    ++kept;
                }
            }
        }
        __syncthreads();
        const double own = tid < a.parts ? segment.above * to_whole + (double)sh.block_mass[tid] : 0.0;
        double upto = own, mass, none = 0.0;
        uint32_t zero = 0, zero_total;
        block_scan<kThreads, 1>(sh, upto, mass, none, zero, zero_total, kept);
        const double target = (double)policy.u * mass;
        const int chosen = block_first<kThreads, 0>(sh, upto > target && own > 0.0, own > 0.0);
        if (tid == chosen) sh.told[0] = fmax(target - (upto - own), 0.0);
        __syncthreads();
        draw<kThreads, kSamplePart / kThreads>(sh, data, weigh, (int64_t)chosen * kSamplePart, kSamplePart, sh.told[0], last);
        tell(a, sh, t, top, policy.tau, shift, mass, full, row.count + kept);
        if (tid == 0) a.row[r].key = last.key, a.row[r].last = last.last;
    }
}

// ---- bits of rows with many kept, and of uncut ones, a workgroup a part -----------------------------------------------------------------------

template <typename DT>
__global__ __launch_bounds__(kPartThreads, 4) void sample_bits_kernel(SampleArgs a, int64_t row0, int64_t rows)
{
    using Entries = PartEntries<DT>;
    constexpr int EPV = Entries::EPV, kVectors = Entries::kVectors;
    for (int64_t i = blockIdx.x; i < rows * a.parts; i += gridDim.x) {
        const int64_t r = i / a.parts, t = row0 + r;
        if (a.row[r].mode != kSampleBin && a.row[r].mode != kSampleDrawn) continue;
        const int64_t begin = (i - r * a.parts) * kSamplePart;
        const int left = (int)min(a.V - begin, (int64_t)kSamplePart);
        Entries z;
        z.load(reinterpret_cast<const char *>(a.z) + (t * a.ld + begin) * DT::kBytes, left);
        const Border last{a.row[r].key, a.row[r].last};
        int32_t *words = a.allowed + t * a.allowed_ld + begin / 32;
#pragma unroll
        for (int v = 0; v < kVectors; ++v) {
            const int e = Entries::first() + v * kWave * EPV;
            float x[EPV];
            unpack<DT>(z.raw[v], x);
            uint32_t word = 0;
#pragma unroll
            for (int k = 0; k < EPV; ++k) word |= (last.keeps(x[k], (int32_t)(begin + e + k)) ? 1u : 0u) << k;
            word <<= e & 31;
#pragma unroll
            for (int off = 1; off < 32 / EPV; off <<= 1) word |= __shfl_xor(word, off, kWave);
            if ((e & 31) == 0 && e < left) words[e >> 5] = (int32_t)word;
        }
    }
}

template <typename DT>
void launch(const SampleArgs &a, hipStream_t s)
{
    for (int64_t row0 = 0; row0 < a.T; row0 += kSampleRows) {
        const int64_t rows = a.T - row0 < kSampleRows ? a.T - row0 : kSampleRows, parts = rows * a.parts;
        const int grid = (int)(parts < (1 << 24) ? parts : 1 << 24);
        // (temperatures of 0 cut, and so may what the other arrays hold)
        if (!a.temperature && !a.top_k && !a.top_p && !a.min_p && !a.allowed && a.parts <= kPartThreads) {
            sample_sums_kernel<DT><<<grid, kPartThreads, 0, s>>>(a, row0, rows);
            sample_uncut_kernel<DT><<<(int)rows, kPartThreads, 0, s>>>(a, row0, rows);
            continue;
        }
        sample_parts_kernel<DT><<<grid, kPartThreads, 0, s>>>(a, row0, rows);
        sample_rows_kernel<DT><<<(int)rows, kThreads, 0, s>>>(a, row0, rows);
        sample_gather_kernel<DT><<<grid, kPartThreads, 0, s>>>(a, row0, rows);
        sample_finish_kernel<DT><<<(int)rows, kThreads, 0, s>>>(a, row0, rows);
        sample_passes_kernel<DT><<<(int)(rows < 512 ? rows : 512), kThreads, 0, s>>>(a, row0, rows);
        if (a.allowed) sample_bits_kernel<DT><<<grid, kPartThreads, 0, s>>>(a, row0, rows);
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
