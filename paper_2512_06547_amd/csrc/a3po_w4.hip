// Products of a few tokens' hidden states with a weight held as 4-bit codes:
//
//   out[t, n] = sum over groups g of scale[n, g] * sum over k in g of (code[n, k] - zero[n, g]) x[t, k]
//
// The weight is read once, straight into registers: 16 bytes a lane are 32 codes of one row, a wavefront holds 16 rows of
// 128 codes (a unit).  Matrix-core products of 16 tokens x 16 rows x 32 codes take float16, in which code - zero is exact: a
// code's bits go into the mantissa of 1,024, and one addition for two codes takes 1,024 + zero off (1,024 + 16 n, for
// the codes that lie four bits higher, leave with a factor of 1/16 in the same instruction).  Hidden values become float16 times
// a power of two of the token's, which brings its largest to between 2^15 and 2^16: bfloat16's eight digits are kept by all that
// are not below 2^-32 of that, and those lose no more than 2^-40 of it.  So products are exact, a group's sum in fp32 is of
// the size of its terms, its scale multiplies it in fp32, and the token's power of two leaves from the output, which is rounded
// once.  (Codes as bfloat16 16 + n with the excess (16 + zero) sum x taken off the sum cost an instruction less for eight, and
// digits: where hidden values are of one sign the sum is many times what is left of it, and errors of 4e-6 came of that, 2e-7 here.)
// With up to 16 tokens the kernel is bound by the weight's bytes, beyond a fixed 6 us for the hidden values and the first codes:
// one token, 1,536 x 151,936 in groups of 128 28 us (4.3 TB/s), 16 tokens, 4,096 x 151,936 in groups of 128 67 (4.9).  With more it is
// the vector instructions, and that they and the matrix instructions take turns rather than overlap, two wavefronts a SIMD that meet
// every two units: 50 tokens, 4,096 x 151,936, fp32 scales of groups of 32 and zero points, 153 us against 92 for the bytes, of
// its cycles vector instructions 61 %, matrix instructions 25 %; a group's scale is a multiply-add for every 32 codes and token.
#include "a3po_common.h"
#include "a3po_direct.h"
#include "a3po_launch.h"

namespace a3po {
namespace {

typedef uint32_t u32x4_half __attribute__((ext_vector_type(4), aligned(2)));

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));

// Constants in registers that the compiler knows nothing of: it would fold them into an instruction each, of which an and-or
// holds one at most.
template <uint32_t VALUE>
__device__ __forceinline__ uint32_t opaque_scalar()
{
    uint32_t v;
    asm("s_mov_b32 %0, %1" : "=s"(v) : "i"(VALUE));
    return v;
}
template <uint32_t VALUE>
__device__ __forceinline__ uint32_t opaque_vector()
{
    uint32_t v;
    asm("v_mov_b32 %0, %1" : "=v"(v) : "i"(VALUE));
    return v;
}

// what a code's zero point takes off two codes: -(1,024 + zero), and -(64 + zero) of those that come as 64 + n
struct Zero {
    f16x2_t low, high;
    __device__ __forceinline__ explicit Zero(uint32_t zero)
    {
        low = __builtin_bit_cast(f16x2_t, (zero | zero << 16) | 0xE400E400u);
        high = low + f16x2_t{(_Float16)960.0f, (_Float16)960.0f};
    }
};
// Codes of a dword, as float16 code - zero, in the order 0 4 1 5 2 6 3 7.
struct Widen {
    uint32_t first = opaque_scalar<0x000F000F>(), second = opaque_scalar<0x00F000F0>(), kilo = opaque_vector<0x64006400>();
    __device__ __forceinline__ f16x8_t operator()(uint32_t d, const Zero &z) const
    {
        const f16x2_t sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
        auto at = [&](uint32_t v, uint32_t mask) { return __builtin_bit_cast(f16x2_t, (v & mask) | kilo); };
        const f16x2_t a = at(d, first) + z.low, b = __builtin_elementwise_fma(at(d, second), sixteenth, z.high);
        const f16x2_t c = at(d >> 8, first) + z.low, e = __builtin_elementwise_fma(at(d >> 8, second), sixteenth, z.high);
        return f16x8_t{a.x, a.y, b.x, b.y, c.x, c.y, e.x, e.y};
    }
};
// the larger magnitude at each place of a pair, as bits
__device__ __forceinline__ uint32_t larger(uint32_t most, const uint4 &v)
{
    u16x2_t m = __builtin_bit_cast(u16x2_t, most);
#pragma unroll
    for (uint32_t w : {v.x, v.y, v.z, v.w}) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2_t, w & 0x7FFF7FFFu));
    return __builtin_bit_cast(uint32_t, m);
}
// the power of two that brings a token whose largest magnitude has these bits to between 2^15 and 2^16
__device__ __forceinline__ int token_shift(uint32_t most) { return most ? 142 - max((int)(most >> 7), 1) : 0; }
// eight hidden values as float16 times that, in the order of the codes
__device__ __forceinline__ uint4 to_halves(const uint4 &v, int shift)
{
    auto low = [&](uint32_t w) { return __builtin_amdgcn_ldexpf(__uint_as_float(w << 16), shift); };
    auto high = [&](uint32_t w) { return __builtin_amdgcn_ldexpf(__uint_as_float(w & 0xFFFF0000u), shift); };
    auto two = [](float a, float b) {
        typedef float f32x2_t __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), f16x2_t));
    };
    return make_uint4(two(low(v.x), low(v.z)), two(high(v.x), high(v.z)), two(low(v.y), low(v.w)), two(high(v.y), high(v.w)));
}

// Lanes l, l + 16, l + 32, l + 48 hold four blocks of 32 codes of one row, a block each; afterwards d[b] of the four lanes
// is block b, a quarter each: what a matrix instruction of that block takes.
__device__ __forceinline__ void transpose_blocks(uint32_t (&d)[4])
{
    auto s0 = __builtin_amdgcn_permlane32_swap(d[0], d[2], false, false);
    auto s1 = __builtin_amdgcn_permlane32_swap(d[1], d[3], false, false);
    auto t0 = __builtin_amdgcn_permlane16_swap(s0[0], s1[0], false, false);
    auto t1 = __builtin_amdgcn_permlane16_swap(s0[1], s1[1], false, false);
    d[0] = t0[0], d[1] = t0[1], d[2] = t1[0], d[3] = t1[1];
}

// Two units of 16 rows are loaded as 8 rows x 128 bytes twice: whole lines, half as many requests as 16 rows x 64 bytes (what
// a compute unit can ask for is counted in lines).  Lane (n, q) of a holds row n % 8, unit n / 8, of b row 8 + n % 8; afterwards
// a is the first unit's row n, b the second's.
__device__ __forceinline__ void sort_units(uint32_t (&a)[4], uint32_t (&b)[4])
{
    constexpr int kRor8 = 0x128;  // lane i of 16 takes lane i - 8
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int x = (int)a[k], y = (int)b[k];
        a[k] = (uint32_t)__builtin_amdgcn_update_dpp(x, y, kRor8, 0xF, 0xC, false);
        b[k] = (uint32_t)__builtin_amdgcn_update_dpp(y, x, kRor8, 0xF, 0x3, false);
    }
}

__device__ __forceinline__ void meet()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(waitcnt_imm(kNoVmWait, 0));
    __builtin_amdgcn_s_barrier();  // (bare: the weight stays in flight)
    asm volatile("" ::: "memory");
}

// BYTES consecutive bytes, at any address
template <int BYTES>
__device__ __forceinline__ void load_run(const char *p, uint32_t (&w)[(BYTES + 3) / 4])
{
    typedef uint32_t v4_t __attribute__((ext_vector_type(4), aligned(1)));
    typedef uint32_t v2_t __attribute__((ext_vector_type(2), aligned(1)));
    typedef uint32_t v1_t __attribute__((aligned(1)));
    typedef uint16_t half_t __attribute__((aligned(1)));
    constexpr int kFours = BYTES / 16, kTwos = BYTES / 8 % 2, kOnes = BYTES / 4 % 2, kRest = BYTES % 4;
#pragma unroll
    for (int i = 0; i < kFours; ++i) {
        const v4_t v = *reinterpret_cast<const v4_t *>(p + 16 * i);
#pragma unroll
        for (int k = 0; k < 4; ++k) w[4 * i + k] = v[k];
    }
    if constexpr (kTwos) {
        const v2_t v = *reinterpret_cast<const v2_t *>(p + 16 * kFours);
        w[4 * kFours] = v.x, w[4 * kFours + 1] = v.y;
    }
    if constexpr (kOnes) w[4 * kFours + 2 * kTwos] = *reinterpret_cast<const v1_t *>(p + 16 * kFours + 8 * kTwos);
    if constexpr (kRest) {
        constexpr int kAt = BYTES - kRest;
        uint32_t v = kRest >= 2 ? *reinterpret_cast<const half_t *>(p + kAt) : 0u;
        if constexpr (kRest & 1) v |= (uint32_t)*reinterpret_cast<const uint8_t *>(p + BYTES - 1) << (8 * (kRest - 1));
        w[BYTES / 4] = v;
    }
}

// ---- few tokens: hidden values resident -------------------------------------------------------------------------------
//
// All hidden values lie in LDS, in the order of the matrix instructions, for as long as the workgroup lives: one workgroup a
// compute unit, sixteen wavefronts.  A set of 16 x (16 / WK) rows is taken at a time: WK wavefronts share the 16 rows, a run of
// UPW units each, and add their sums through LDS.  A wavefront's weight is loaded NB sets ahead into registers (four units or
// more in flight, 64 KiB and more a compute unit) and waits for nobody else's.

// a row's codes of UPW units in a row, with their scales and zero points
template <int UPW, int GROUP, bool ZEROS, bool SCALE_F32>
struct Run {
    static constexpr int kGroups = UPW * 128 / GROUP, kScaleBytes = kGroups * (SCALE_F32 ? 4 : 2);
    u32x4_t codes[UPW];
    uint32_t scales[(kScaleBytes + 3) / 4], zeros[ZEROS ? (kGroups + 3) / 4 : 1];
    // c: the block's first row and unit; a, b: a lane's place in pairs of units (see sort_units), one: in a single unit
    __device__ __forceinline__ void load(const char *c, uint32_t a, uint32_t b, uint32_t one, const char *s, const char *z)
    {
#pragma unroll
        for (int u = 0; u + 1 < UPW; u += 2) {
            codes[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(c + u * 64 + a));
            codes[u + 1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(c + u * 64 + b));
        }
        if constexpr (UPW % 2) codes[UPW - 1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(c + (UPW - 1) * 64 + one));
        load_run<kScaleBytes>(s, scales);
        if constexpr (ZEROS) load_run<kGroups>(z, zeros);
    }
    __device__ __forceinline__ float scale(int g) const
    {
        if constexpr (SCALE_F32) return __uint_as_float(scales[g]);
        else return __uint_as_float(g & 1 ? scales[g / 2] & 0xFFFF0000u : scales[g / 2] << 16);
    }
    __device__ __forceinline__ Zero zero(int g) const { return Zero(ZEROS ? zeros[g / 4] >> (8 * (g % 4)) & 0xFFu : 8u); }
};

template <int MT, int UPW, int NB, int GROUP, bool ZEROS, bool SCALE_F32>
__global__ __launch_bounds__(1024) void w4_resident_kernel(W4Args a, int wk_shift, int tp_shift, int sets)
{
    constexpr int S = 128 / GROUP, BLOCKS = GROUP / 32, kAll = 16;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int n16 = lane & 15, q = lane >> 4;
    const int WK = 1 << wk_shift, WR = kAll >> wk_shift, wk = wave & (WK - 1), wr = wave >> wk_shift;
    static_assert(MT <= 2, "tokens are a power of two");
    const int tps = MT > 1 ? 5 : tp_shift, TP = 1 << tps;
    // (the last wavefronts' runs move down to end with the row; units that another one has as well count for nothing here)
    const int units = a.H >> 7, u0 = min(wk * UPW, units - UPW), skip = wk * UPW - u0;
    const int64_t groups = a.H / GROUP, row_bytes = a.H / 2;
    char *xs = lds;                                          // [units][4][4][TP] 16 bytes
    char *red = lds + (size_t)a.H * TP * 2;                  // [16 wavefronts][MT][64] 16 bytes
    int *shifts = reinterpret_cast<int *>(red + 16 * 1024 * MT);  // [TP]

    // lane offsets from a set's first row (fewer than 16 rows in all: the last one again)
    const uint32_t row_lane = (uint32_t)min((int64_t)n16, a.V - 1);
    const uint32_t one_lane = row_lane * (uint32_t)row_bytes + q * 16, group_lane = row_lane * (uint32_t)groups;
    auto pair_lane = [&](int row) { return (uint32_t)min((int64_t)row, a.V - 1) * (uint32_t)row_bytes + (n16 >> 3) * 64 + q * 16; };
    const uint32_t a_lane = pair_lane(n16 & 7), b_lane = pair_lane(8 + (n16 & 7));
    constexpr uint32_t kScale = SCALE_F32 ? 4 : 2;
    Run<UPW, GROUP, ZEROS, SCALE_F32> run[NB];
    // first row of this wavefront's block in a set; the last block moves up to end with the weight
    auto first_row = [&](int set) { return min(((int64_t)set * WR + wr) * 16, max(a.V - 16, (int64_t)0)); };
    // (no branch around the loads: at one the compiler waits for all that are in flight; sets beyond the last are the last)
    auto fetch = [&](int set, Run<UPW, GROUP, ZEROS, SCALE_F32> &to) {
        const int64_t row = first_row(min(set, sets - 1));
        const char *codes = reinterpret_cast<const char *>(a.codes) + row * row_bytes + u0 * 64;
        const int64_t group = row * groups + u0 * S;
        to.load(codes, a_lane, b_lane, one_lane, static_cast<const char *>(a.scales) + group * kScale + group_lane * kScale,
                ZEROS ? reinterpret_cast<const char *>(a.zeros) + group + group_lane : nullptr);
        __builtin_amdgcn_sched_barrier(0);  // (in this order: what is waited for first is issued first)
    };
    // The hidden values first, then the weight: what is asked for later arrives later, and those would be waited for with all of
    // the weight that is in flight.  A thread's pieces, eight values each, are all one token's: piece i is the row's k8_of(i)-th.
    // (Threads beyond the last token have that one again; their products are not stored.)
    const int eights = units * 16, token = (int)threadIdx.x & (TP - 1), most_pieces = (eights + (1024 >> tps) - 1) >> (10 - tps);
    auto k8_of = [&](int i) { return ((int)threadIdx.x >> tps) + (i << (10 - tps)); };
    const char *x_row = static_cast<const char *>(a.x) + min((int64_t)token, a.T - 1) * a.ldx * 2;
    auto load_x = [&](int i) {
        const u32x4_half h = *reinterpret_cast<const u32x4_half *>(x_row + min(k8_of(i), eights - 1) * 16);
        return make_uint4(h.x, h.y, h.z, h.w);
    };
    auto place_x = [&](int i) {
        const int k8 = k8_of(i);
        // groups of a whole unit: the lanes of a block of codes keep it, and the quarter of the unit that they multiply is theirs
        const int at = GROUP == 128 ? (k8 & ~15) | (k8 & 3) << 2 | (k8 >> 2 & 3) : k8;
        return reinterpret_cast<uint4 *>(xs + ((at << tps) + token) * 16);
    };
    // Four a thread, and four more, two at a time, where rows are long (eight always: 1 x 896 0.5 us more, 16 x 2,048 1.2; the longer
    // rows' behind the weight: 16 x 4,096 2.5 more).
    constexpr int kPieces = 8;  // (w4_resident lets no more in)
    uint4 mine[kPieces];
#pragma unroll
    for (int i = 0; i < 4; ++i) mine[i] = load_x(i);
    if (most_pieces > 4) mine[4] = load_x(4), mine[5] = load_x(5);
    if (most_pieces > 6) mine[6] = load_x(6), mine[7] = load_x(7);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int b = 0; b < NB; ++b) fetch((int)blockIdx.x + b * (int)gridDim.x, run[b]);
    // the token's largest value: of this thread's, the wavefront's, all sixteen's (pieces beyond the row are its last again)
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) most = larger(most, mine[i]);
    if (most_pieces > 4) most = larger(larger(most, mine[4]), mine[5]);
    if (most_pieces > 6) most = larger(larger(most, mine[6]), mine[7]);
    most = max(most & 0xFFFFu, most >> 16);
    for (int off = TP; off < kWave; off <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off, kWave));
    if (lane < TP) reinterpret_cast<uint32_t *>(red)[wave * TP + lane] = most;
    meet();
#pragma unroll
    for (int w = 0; w < kAll; ++w) most = max(most, reinterpret_cast<const uint32_t *>(red)[w * TP + token]);
    const int shift = token_shift(most);
    if ((int)threadIdx.x < TP) shifts[threadIdx.x] = shift;
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
        if (k8_of(i) < eights) *place_x(i) = to_halves(mine[i], shift);
    meet();

    const Widen widen;
    // (with fewer than 16 tokens the lanes of the others read these again; their products are not stored)
    const char *x_lane = xs + (q * TP + (n16 & (TP - 1))) * 16;

    auto multiply = [&](const Run<UPW, GROUP, ZEROS, SCALE_F32> &from, f32x4_t (&acc)[MT]) {
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[m] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        uint32_t codes[UPW][4];
#pragma unroll
        for (int u = 0; u < UPW; ++u)
#pragma unroll
            for (int k = 0; k < 4; ++k) codes[u][k] = from.codes[u][k];
#pragma unroll
        for (int u = 0; u + 1 < UPW; u += 2) sort_units(codes[u], codes[u + 1]);
#pragma unroll
        for (int u = 0; u < UPW; ++u) {
            uint32_t(&d)[4] = codes[u];
            if constexpr (GROUP < 128) transpose_blocks(d);
            const char *x = x_lane + (size_t)(u0 + u) * 16 * TP * 16;
            f32x4_t part[MT];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int gi = g / BLOCKS;
                const f16x8_t wide = widen(d[g], from.zero(u * S + gi));
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    part[m] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                        *reinterpret_cast<const f16x8_t *>(x + ((size_t)g * 4 * TP + m * 16) * 16), wide,
                        g % BLOCKS == 0 ? f32x4_t{0.0f, 0.0f, 0.0f, 0.0f} : part[m], 0, 0, 0);
                if (g % BLOCKS == BLOCKS - 1) {
                    const float scale = u < skip ? 0.0f : from.scale(u * S + gi);
#pragma unroll
                    for (int m = 0; m < MT; ++m) acc[m] += part[m] * scale;
                }
            }
        }
    };
    auto put_out = [&](int64_t t, int64_t n, float v) {
        if (a.out_dt == A3PO_F32) static_cast<float *>(a.out)[t * a.ldo + n] = v;
        else store_elem<Bf16>(a.out, t * a.ldo + n, v);
    };
    auto finish = [&](int set, f32x4_t (&acc)[MT]) {
        meet();  // (the sums of the set before are read)
#pragma unroll
        for (int m = 0; m < MT; ++m) *reinterpret_cast<f32x4_t *>(red + ((wave * MT + m) * kWave + lane) * 16) = acc[m];
        meet();
        for (int o = threadIdx.x; o < WR * MT * 256; o += 1024) {
            const int block = o / (MT * 256), token = o / 16 % (MT * 16), n = o & 15;
            if (token >= a.T) continue;
            const char *from = red + (((block << wk_shift) * MT + token / 16) * kWave + (token / 4 % 4) * 16 + n) * 16 + token % 4 * 4;
            constexpr int kFrom = MT * kWave * 16;
            float total = 0.0f;
            for (int k = 0; k < WK; k += 4) {  // (four reads in flight; beyond the last wavefront its sum again, for nothing)
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const float *>(from + min(k + j, WK - 1) * kFrom);
#pragma unroll
                for (int j = 0; j < 4; ++j) total += k + j < WK ? v[j] : 0.0f;
            }
            const int64_t want = ((int64_t)set * WR + block) * 16, row = min(want, max(a.V - 16, (int64_t)0)) + n;
            if (row >= want && row < a.V) put_out(token, row, __builtin_amdgcn_ldexpf(total, -shifts[token]));
        }
    };

    const int step = (int)gridDim.x;
    int set = blockIdx.x, left = (sets - 1 - set) / step + 1;
    for (; left >= NB; left -= NB)
#pragma unroll
        for (int b = 0; b < NB; ++b, set += step) {
            f32x4_t acc[MT];
            multiply(run[b], acc);
            fetch(set + NB * step, run[b]);
            finish(set, acc);
        }
#pragma unroll
    for (int b = 0; b < NB - 1; ++b, set += step)
        if (b < left) {
            f32x4_t acc[MT];
            multiply(run[b], acc);
            finish(set, acc);
        }
}

// ---- more tokens, long or odd rows: hidden values stream through LDS ----------------------------------------------------
//
// A first kernel writes the hidden values as float16 in the order of the matrix instructions, so that the second copies them to
// LDS as they are: [pass of 16 MT tokens][unit][4 blocks of codes][MT][64 lanes] 16 bytes, then the tokens' powers of
// two.  Units are a multiple of four, those beyond the row hold zeros (a branch around them would cost the wait that loads
// are kept out of branches for).

constexpr int unit_bytes(int mt) { return kW4UnitBytes * mt; }

// a workgroup takes a token (those beyond the last are zeros); what it has no registers for it reads again
template <int MT>
__global__ __launch_bounds__(256) void w4_order_kernel(W4Args a, char *to, int units, int *shifts)
{
    constexpr int kFirst = 2;
    __shared__ uint32_t red[256 / kWave];
    const int64_t token = blockIdx.x, pass = token / (16 * MT);
    const int in_pass = (int)(token % (16 * MT)), pieces = units * 16;
    const char *row = static_cast<const char *>(a.x) + token * a.ldx * 2;
    auto load = [&](int p) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (token < a.T && p * 8 < a.H) {
            const u32x4_half h = *reinterpret_cast<const u32x4_half *>(row + (int64_t)p * 16);
            v = make_uint4(h.x, h.y, h.z, h.w);
        }
        return v;
    };
    uint4 first[kFirst];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < kFirst; ++i) first[i] = load(threadIdx.x + i * 256);
#pragma unroll
    for (int i = 0; i < kFirst; ++i) most = larger(most, first[i]);
    for (int p = threadIdx.x + kFirst * 256; p < pieces; p += 256) most = larger(most, load(p));
    most = max(most & 0xFFFFu, most >> 16);
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off, kWave));
    if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x / kWave] = most;
    __syncthreads();
#pragma unroll
    for (uint32_t m : red) most = max(most, m);
    const int shift = token_shift(most);
    if (threadIdx.x == 0) shifts[token] = shift;
    auto keep = [&](int p, const uint4 &v) {
        if (p < pieces)
            *reinterpret_cast<uint4 *>(to + (pass * units + (p >> 4)) * unit_bytes(MT) +
                                       (((p >> 2 & 3) * MT + in_pass / 16) * kWave + (p & 3) * 16 + in_pass % 16) * 16) =
                to_halves(v, shift);
    };
#pragma unroll
    for (int i = 0; i < kFirst; ++i) keep(threadIdx.x + i * 256, first[i]);
    for (int p = threadIdx.x + kFirst * 256; p < pieces; p += 256) keep(p, load(p));
}

// arrays of scales or zero points too short for the loads of the second kernel, with zeros behind them
__global__ __launch_bounds__(kW4ShortBytes) void w4_short_kernel(const uint8_t *from, int bytes, uint8_t *to)
{
    to[threadIdx.x] = (int)threadIdx.x < bytes ? from[threadIdx.x] : 0;
}

// 16 bytes of an array, `over` of which would lie behind its end: loaded that much earlier, the others moved to the front
__device__ __forceinline__ u32x4_t load_piece(const char *p)
{
    typedef uint32_t v4_t __attribute__((ext_vector_type(4), aligned(1)));
    return *reinterpret_cast<const v4_t *>(p);
}
__device__ __forceinline__ u32x4_t move_piece(u32x4_t v, int over)
{
    if (__any(over > 0)) {
        uint64_t lo = (uint64_t)v.y << 32 | v.x, hi = (uint64_t)v.w << 32 | v.z;
        const int bits = min(over, 15) * 8;
        if (over >= 8) {
            lo = hi >> (bits - 64);
            hi = 0;
        } else if (over > 0) {
            lo = lo >> bits | hi << (64 - bits);
            hi >>= bits;
        }
        v.x = (uint32_t)lo, v.y = (uint32_t)(lo >> 32), v.z = (uint32_t)hi, v.w = (uint32_t)(hi >> 32);
    }
    return v;
}

// The blocks of scales (64 bytes of a row at a time) and zero points that a wavefront's 16 R rows need for the next
// units: from memory into registers, from there into the wavefront's own LDS.
template <int R, int GROUP, bool ZEROS, bool SCALE_F32>
struct GroupBlocks {
    static constexpr int S = 128 / GROUP, kBytes = SCALE_F32 ? 4 : 2, kBlock = 64, kUnits = kBlock / (S * kBytes), kZeroBytes = kUnits * S;
    static constexpr int kLanes = kBlock / 16, kTogether = kWave / kLanes;  // lanes a row, rows a load
    static constexpr int kStride = kBlock + 16, kZeroStride = kZeroBytes + 16;  // (rows on different banks)
    static constexpr int kLds = 32 * (kStride + (ZEROS ? kZeroStride : 0));
    static constexpr int kPieces = 16 * R / kTogether, kZeroLanes = kZeroBytes / 16, kZeroPieces = (16 * R * kZeroLanes + kWave - 1) / kWave;
    u32x4_t s[kPieces], z[kZeroPieces];

    // a row's bytes, the block's first byte of the wavefront's first row, and how far a piece may begin from there
    struct Place {
        const char *from;
        int last;
    };
    __device__ __forceinline__ static Place place(const void *array, int64_t array_rows, int64_t row, int row_len, int64_t at)
    {
        Place p;
        p.from = static_cast<const char *>(array) + row * row_len + at;
        p.last = (int)min(array_rows * row_len - 16 - (row * row_len + at), (int64_t)0x7FFFFFFF);
        return p;
    }
    __device__ __forceinline__ static int lane_at(int row, int rows, int row_len, int byte) { return min(row, rows - 1) * row_len + byte; }

    // row, rows: the wavefront's first row and their number; groups: of a row
    __device__ __forceinline__ void fetch(const W4Args &a, int64_t row, int rows, int groups, int block, int lane)
    {
        const Place p = place(a.scales, a.V, row, groups * kBytes, (int64_t)block * kBlock);
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            s[i] = load_piece(p.from + min(lane_at(i * kTogether + lane / kLanes, rows, groups * kBytes, lane % kLanes * 16), p.last));
        if constexpr (ZEROS) {
            const Place zp = place(a.zeros, a.V, row, groups, (int64_t)block * kZeroBytes);
#pragma unroll
            for (int i = 0; i < kZeroPieces; ++i)
                z[i] = load_piece(zp.from + min(lane_at(i * (kWave / kZeroLanes) + lane / kZeroLanes, rows, groups, lane % kZeroLanes * 16), zp.last));
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    __device__ __forceinline__ void store(const W4Args &a, char *lds, int64_t row, int rows, int groups, int block, int lane)
    {
        const int row_bytes = groups * kBytes;
        const Place p = place(a.scales, a.V, row, row_bytes, (int64_t)block * kBlock);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            u32x4_t v = move_piece(s[i], lane_at(i * kTogether + lane / kLanes, rows, row_bytes, lane % kLanes * 16) - p.last);
            if ((block + 1) * kBlock > row_bytes) {  // what lies behind the row's end is another row's: no scale at all here
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int left = row_bytes - (block * kBlock + lane % kLanes * 16 + 4 * k);
                    v[k] = left >= 4 ? v[k] : left == 2 ? v[k] & 0xFFFFu : 0u;
                }
            }
            lds_put(lds + (i * kTogether + lane / kLanes) * kStride + lane % kLanes * 16, v);
        }
        if constexpr (ZEROS) {
            const Place zp = place(a.zeros, a.V, row, groups, (int64_t)block * kZeroBytes);
#pragma unroll
            for (int i = 0; i < kZeroPieces; ++i) {
                const int r = i * (kWave / kZeroLanes) + lane / kZeroLanes;
                const u32x4_t v = move_piece(z[i], lane_at(r, rows, groups, lane % kZeroLanes * 16) - zp.last);
                if (r < 16 * R) lds_put(lds + 32 * kStride + r * kZeroStride + lane % kZeroLanes * 16, v);
            }
        }
    }
    // of row r, unit u of the block
    __device__ __forceinline__ static void scales(const char *lds, int r, int u, float (&out)[S])
    {
        const char *p = lds + r * kStride + u * (S * kBytes);
        if constexpr (SCALE_F32) {
            typedef float v_t __attribute__((ext_vector_type(S > 1 ? S : 2)));
            if constexpr (S == 1) out[0] = lds_get<float>(p);
            else {
                const v_t v = lds_get<v_t>(p);
#pragma unroll
                for (int g = 0; g < S; ++g) out[g] = v[g];
            }
        } else {
            uint32_t w[(S + 1) / 2];
            if constexpr (S == 1) w[0] = lds_get<uint16_t>(p);
            else
#pragma unroll
                for (int k = 0; k < S / 2; ++k) w[k] = lds_get<uint32_t>(p + 4 * k);
#pragma unroll
            for (int g = 0; g < S; ++g) out[g] = __uint_as_float(g & 1 ? w[g / 2] & 0xFFFF0000u : w[g / 2] << 16);
        }
    }
    __device__ __forceinline__ static Zero zero(const char *lds, int r, int u, int g)
    {
        return Zero(ZEROS ? lds_get<uint8_t>(lds + 32 * kStride + r * kZeroStride + u * S + g) : 8u);
    }
};

// Eight wavefronts of 16 R rows each, tile after tile.  Two units a chunk: chunk c is multiplied from LDS while chunks c + 1 and
// c + 2 of the hidden values arrive in LDS (direct loads) and of the codes in registers, the next tile's among them.  What is
// waited for before a barrier is counted by hand: everything but the operations issued behind the next chunk's direct loads.
template <int MT, int R, int GROUP, bool ZEROS, bool SCALE_F32>
__device__ __forceinline__ void stream_tiles(const W4Args &a, const char *x, int units, int64_t first_row, int tiles, int64_t t0, char *xs,
                                             char *own, const int *shifts)
{
    constexpr int UC = 2, S = 128 / GROUP, BLOCKS = GROUP / 32, kChunk = UC * unit_bytes(MT), kRows = 8 * 16 * R;
    constexpr int kCopies = kChunk / 8192;                          // direct loads of 1 KiB a wavefront and chunk
    static_assert(kChunk % 8192 == 0, "whole loads");
    constexpr int kBehind = UC * R + kCopies + UC * R;              // operations behind the next chunk's
    using Groups = GroupBlocks<R, GROUP, ZEROS, SCALE_F32>;
    constexpr int kPerBlock = Groups::kUnits / UC;  // chunks of a block of scales
    static_assert(kPerBlock % 2 == 0, "chunks go in pairs");
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int n16 = lane & 15, q = lane >> 4, step = (int)gridDim.x;
    const int chunks = units / UC, groups = a.H / GROUP, row_bytes = a.H / 2;
    const int mine = tiles > (int)blockIdx.x ? (tiles - 1 - (int)blockIdx.x) / step + 1 : 0;
    if (mine == 0) return;
    // rows of this wavefront in its i-th tile; those beyond the last move up to end with the weight
    const int rows = (int)min((int64_t)(16 * R), a.V);
    auto wanted = [&](int i) { return first_row + ((int64_t)blockIdx.x + (int64_t)i * step) * kRows + wave * (16 * R); };
    auto row_of = [&](int i) { return min(wanted(i), max(a.V - 16 * R, (int64_t)0)); };
    uint32_t a_lane[R], b_lane[R];
    const uint32_t in_row = (n16 >> 3) * 64 + q * 16;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        a_lane[r] = (uint32_t)min(r * 16 + (n16 & 7), rows - 1) * (uint32_t)row_bytes;
        b_lane[r] = (uint32_t)min(r * 16 + 8 + (n16 & 7), rows - 1) * (uint32_t)row_bytes;
    }
    struct Chunk {
        u32x4_t w[UC * R];
    };
    // the place of what is fetched next: tile, chunk
    auto advance = [&](int &i, int &c) {
        ++c;
        const bool over = c == chunks;
        c = over ? 0 : c;
        i = over ? min(i + 1, mine - 1) : i;  // (beyond the last tile it is the last again: no branch around loads, at one the
    };                                        // compiler waits for all that are in flight)
    int wi = 0, wc = 0, xc = 0;
    auto fetch_w = [&](Chunk &to) {
        const char *codes = reinterpret_cast<const char *>(a.codes) + row_of(wi) * row_bytes;
        // (a row that ends inside the pair of units: its last 16 bytes again, against hidden values of zero)
        const uint32_t at = min(wc * 128 + in_row, (uint32_t)row_bytes - 16);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            to.w[2 * r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(codes + (a_lane[r] + at)));
            to.w[2 * r + 1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(codes + (b_lane[r] + at)));
        }
        advance(wi, wc);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    const __amdgpu_buffer_rsrc_t x_buffer = dma_buffer(x, (uint32_t)(units * unit_bytes(MT)));
    auto fetch_x = [&](int to) {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int at = i * 8192 + wave * 1024;
            dma16(x_buffer, lane * 16, (uint32_t)(xc * kChunk + at), xs + to * kChunk + at);
        }
        xc = xc + 1 == chunks ? 0 : xc + 1;
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    // blocks of scales: the one in registers
    Groups next;
    int gi = 0, gb = 0;
    const int blocks = (chunks + kPerBlock - 1) / kPerBlock;
    auto fetch_groups = [&]() { next.fetch(a, row_of(gi), rows, groups, gb, lane); };
    auto store_groups = [&]() {
        next.store(a, own, row_of(gi), rows, groups, gb, lane);
        gb = gb + 1 == blocks ? 0 : gb + 1;
        gi = gb == 0 ? min(gi + 1, mine - 1) : gi;
    };

    const Widen widen;
    f32x4_t acc[R][MT];
    auto clear = [&]() {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[r][m] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    };
    // (a chunk's registers are free for the next but one as soon as its lanes are sorted)
    auto sort = [&](const Chunk &from, uint32_t (&d)[R][UC][4]) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int i = 0; i < UC; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) d[r][i][k] = from.w[2 * r + i][k];
            sort_units(d[r][0], d[r][1]);
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    auto multiply = [&](int which, int in_block, uint32_t (&d)[R][UC][4]) {
#pragma unroll
        for (int i = 0; i < UC; ++i) {
            const char *unit = xs + which * kChunk + i * unit_bytes(MT);
            float scale[R][S];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                transpose_blocks(d[r][i]);
                Groups::scales(own, r * 16 + n16, in_block * UC + i, scale[r]);
            }
            f32x4_t part[R][MT];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f16x8_t wide[R];
#pragma unroll
                for (int r = 0; r < R; ++r) wide[r] = widen(d[r][i][g], Groups::zero(own, r * 16 + n16, in_block * UC + i, g / BLOCKS));
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const f16x8_t xv = lds_get<f16x8_t>(unit + ((g * MT + m) * kWave + lane) * 16);
#pragma unroll
                    for (int r = 0; r < R; ++r)
                        part[r][m] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                            xv, wide[r], g % BLOCKS == 0 ? f32x4_t{0.0f, 0.0f, 0.0f, 0.0f} : part[r][m], 0, 0, 0);
                }
                // (behind the products of all tokens: a sum that is read at once holds the wavefront up for its whole length)
                if (g % BLOCKS == BLOCKS - 1)
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int r = 0; r < R; ++r) acc[r][m] += part[r][m] * scale[r][g / BLOCKS];
            }
        }
    };
    auto put_out = [&](int i) {
        const int64_t want = wanted(i), at = row_of(i);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            typedef int i32x4_t __attribute__((ext_vector_type(4)));
            const i32x4_t shift = lds_get<i32x4_t>(shifts + m * 16 + q * 4);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[r][m][k] = __builtin_amdgcn_ldexpf(acc[r][m][k], -shift[k]);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t n = at + r * 16 + n16;
            if (n < want || n >= a.V) continue;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int64_t t = t0 + m * 16 + q * 4 + k;
                    if (t < a.T) {
                        if (a.out_dt == A3PO_F32) static_cast<float *>(a.out)[t * a.ldo + n] = acc[r][m][k];
                        else store_elem<Bf16>(a.out, t * a.ldo + n, acc[r][m][k]);
                    }
                }
        }
    };

    int tile = 0, c = 0, in_block = 0;
    const int64_t total = (int64_t)mine * chunks;
    auto meet_next = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(waitcnt_imm(kBehind, 0));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    int which = 0;  // the third of the hidden values' LDS that is multiplied
    auto one = [&](Chunk &now) {
        uint32_t d[R][UC][4];
        sort(now, d);
        fetch_x(which == 0 ? 2 : which - 1);
        fetch_w(now);
        multiply(which, in_block, d);
        which = which == 2 ? 0 : which + 1;
        ++in_block;
        ++c;
    };
    Chunk k0, k1;
    meet();  // (the tiles before these are read)
    fetch_groups();
    fetch_x(0);
    fetch_w(k0);
    fetch_x(1);
    fetch_w(k1);
    clear();
    meet_next();
    for (int64_t s = 0; s < total; s += 2) {
        if (in_block == 0) {
            store_groups();
            fetch_groups();
        }
        one(k0);
        meet_next();
        one(k1);
        if (in_block == kPerBlock) in_block = 0;
        if (c == chunks) {
            put_out(tile);
            clear();
            ++tile;
            c = in_block = 0;
        }
        meet_next();
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, 0));  // (nothing may arrive in LDS that the next tiles, or workgroup, use)
}

// Tiles of 256 rows first, then a last round of 128 rows where no more are left for it: a compute unit is done with those in
// half the time.
template <int MT, int GROUP, bool ZEROS, bool SCALE_F32>
__global__ __launch_bounds__(512) void w4_stream_kernel(W4Args a, const char *ordered, const int *token_shifts, int units, int wide_tiles,
                                                        int narrow_tiles)
{
    constexpr int kOwn = GroupBlocks<2, GROUP, ZEROS, SCALE_F32>::kLds;
    extern __shared__ __align__(16) char lds[];
    int *shifts = reinterpret_cast<int *>(lds + 6 * unit_bytes(MT));  // of this pass' tokens
    char *own = lds + 6 * unit_bytes(MT) + 64 * MT + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * kOwn;
    const uint32_t pass = __builtin_amdgcn_readfirstlane(blockIdx.y);  // (or the loads' descriptor ends up in vector registers)
    if (threadIdx.x < 16 * MT) shifts[threadIdx.x] = token_shifts[pass * (16 * MT) + threadIdx.x];  // (read behind barriers)
    const char *x = ordered + (int64_t)pass * units * unit_bytes(MT);
    const int64_t t0 = (int64_t)pass * (16 * MT);
    stream_tiles<MT, 2, GROUP, ZEROS, SCALE_F32>(a, x, units, 0, wide_tiles, t0, lds, own, shifts);
    stream_tiles<MT, 1, GROUP, ZEROS, SCALE_F32>(a, x, units, (int64_t)wide_tiles * 256, narrow_tiles, t0, lds, own, shifts);
}

template <int MT, int GROUP, bool ZEROS, bool SCALE_F32>
hipError_t launch_stream(W4Args a, void *workspace, int cus, hipStream_t s)
{
    static LdsLimitState lds_limit;
    auto *kernel = w4_stream_kernel<MT, GROUP, ZEROS, SCALE_F32>;
    if (const hipError_t e = ensure_lds_limit(reinterpret_cast<const void *>(kernel), kW4MaxLds, lds_limit)) return e;
    const int units = (a.H + 511) / 512 * 4;
    const unsigned passes = (unsigned)((a.T + 16 * MT - 1) / (16 * MT));
    char *ordered = static_cast<char *>(workspace);
    int *shifts = reinterpret_cast<int *>(ordered + (size_t)passes * units * unit_bytes(MT));
    w4_order_kernel<MT><<<dim3(passes * (16 * MT)), dim3(256), 0, s>>>(a, ordered, units, shifts);
    if (const hipError_t e = hipGetLastError()) return e;
    // scales and zero points are loaded 16 bytes at a time: short arrays from a copy behind the hidden values
    uint8_t *spare = reinterpret_cast<uint8_t *>(shifts + passes * (16 * MT));
    const int64_t groups = a.V * (a.H / GROUP), bytes = groups * (SCALE_F32 ? 4 : 2);
    if (bytes < 16) {
        w4_short_kernel<<<1, kW4ShortBytes, 0, s>>>(static_cast<const uint8_t *>(a.scales), (int)bytes, spare);
        if (const hipError_t e = hipGetLastError()) return e;
        a.scales = spare;
    }
    if (ZEROS && groups < 16) {
        w4_short_kernel<<<1, kW4ShortBytes, 0, s>>>(a.zeros, (int)groups, spare + kW4ShortBytes);
        if (const hipError_t e = hipGetLastError()) return e;
        a.zeros = spare + kW4ShortBytes;
    }
    const W4Tiles p = w4_tiles(a.V, cus);
    const int lds = 6 * unit_bytes(MT) + 64 * MT + 8 * GroupBlocks<2, GROUP, ZEROS, SCALE_F32>::kLds;
    kernel<<<dim3((unsigned)p.blocks, passes), dim3(512), lds, s>>>(a, ordered, shifts, units, p.wide, p.narrow);
    return hipGetLastError();
}

template <int MT, int UPW, int NB, int GROUP, bool ZEROS, bool SCALE_F32>
hipError_t launch_resident(const W4Args &a, const W4Plan &p, hipStream_t s)
{
    static LdsLimitState lds_limit;
    auto *kernel = w4_resident_kernel<MT, UPW, NB, GROUP, ZEROS, SCALE_F32>;
    if (const hipError_t e = ensure_lds_limit(reinterpret_cast<const void *>(kernel), kW4MaxLds, lds_limit)) return e;
    kernel<<<dim3((unsigned)p.blocks), dim3(1024), p.lds, s>>>(a, p.wk_shift, p.tp_shift, p.sets);
    return hipGetLastError();
}

template <int MT, int GROUP, bool ZEROS, bool SCALE_F32>
hipError_t launch_units(const W4Args &a, const W4Plan &p, hipStream_t s)
{
    // Two sets ahead are enough, and a third costs the registers that keep addresses: 1 x 1,536 x 151,936, us, three / two: groups of
    // 32 bf16 with zero points 48 (spilled) / 38, of 64 31 / 28, of 128 31 / 29.
    if (p.units == 2) return launch_resident<MT, 2, 2, GROUP, ZEROS, SCALE_F32>(a, p, s);
    if (p.units == 3) return launch_resident<MT, 3, 2, GROUP, ZEROS, SCALE_F32>(a, p, s);
    if constexpr (GROUP > 32 || !SCALE_F32) return launch_resident<MT, 4, 2, GROUP, ZEROS, SCALE_F32>(a, p, s);
    return hipErrorInvalidValue;  // (w4_plan gives no such call four units)
}

template <int GROUP, bool ZEROS, bool SCALE_F32>
hipError_t launch_tokens(const W4Args &a, void *workspace, hipStream_t s)
{
    const GemmGrid chip = gemm_grid();
    const int cus = chip.nxcd * chip.per_xcd;
    const W4Plan p = w4_plan(a.T, a.H, a.V, a.group, SCALE_F32, cus);
    if (p.units && p.blocks16 == 1) return launch_units<1, GROUP, ZEROS, SCALE_F32>(a, p, s);
    if (p.units) return launch_units<2, GROUP, ZEROS, SCALE_F32>(a, p, s);
    // (more than 64 tokens: shared out evenly among as many readings of the weight as 64 at a time take)
    const int64_t passes = (a.T + 63) / 64, tokens = (a.T + passes - 1) / passes;
    if (tokens <= 16) return launch_stream<1, GROUP, ZEROS, SCALE_F32>(a, workspace, cus, s);
    if (tokens <= 32) return launch_stream<2, GROUP, ZEROS, SCALE_F32>(a, workspace, cus, s);
    if (tokens <= 48) return launch_stream<3, GROUP, ZEROS, SCALE_F32>(a, workspace, cus, s);
    return launch_stream<4, GROUP, ZEROS, SCALE_F32>(a, workspace, cus, s);
}

template <int GROUP>
hipError_t launch_group(const W4Args &a, void *ws, hipStream_t s)
{
    const bool f32 = a.scale_dt == A3PO_F32;
    if (a.zeros) return f32 ? launch_tokens<GROUP, true, true>(a, ws, s) : launch_tokens<GROUP, true, false>(a, ws, s);
    return f32 ? launch_tokens<GROUP, false, true>(a, ws, s) : launch_tokens<GROUP, false, false>(a, ws, s);
}

}  // namespace

hipError_t launch_w4_linear(const W4Args &a, void *workspace, hipStream_t s)
{
    if (a.group == 32) return launch_group<32>(a, workspace, s);
    if (a.group == 64) return launch_group<64>(a, workspace, s);
    return launch_group<128>(a, workspace, s);
}

}  // namespace a3po
