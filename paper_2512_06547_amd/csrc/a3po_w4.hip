// Products of a few tokens' hidden states with a weight held as 4-bit codes:
//
//   out[t, n] = sum over groups g of scale[n, g] * sum over k in g of (code[n, k] - zero[n, g]) x[t, k]
//
// The weight is read once, straight into registers: 16 bytes a lane are 32 codes of one row, a wavefront holds 16 rows of
// 128 codes (a unit).  A code n becomes the bfloat16 16 + n by putting its bits into the mantissa of 16 (one shift and one
// and-or for two codes), so that matrix-core products of 16 tokens x 16 rows x 32 codes take it exactly; the excess
// (16 + zero) * sum x is what the fp32 accumulator of a group starts from, and the group's scale multiplies the sum.
// Products are exact, sums are fp32, the output is rounded once.
// With up to 16 tokens the kernel is bound by the weight's bytes: the matrix cores take a seventh of that time.
#include "a3po_common.h"
#include "a3po_direct.h"
#include "a3po_launch.h"

namespace a3po {
namespace {

constexpr int kWaves = kW4Waves, kThreads = kWaves * kWave;

typedef uint32_t u32x4_half __attribute__((ext_vector_type(4), aligned(2)));

// codes of dword d, as bfloat16 16 + n, in the order 0 4 1 5 2 6 3 7
__device__ __forceinline__ bf16x8_t widen(uint32_t d)
{
    constexpr uint32_t kMask = 0x00780078u, kSixteen = 0x41804180u;
    const u32x4_t w = {((d << 3) & kMask) | kSixteen, ((d >> 1) & kMask) | kSixteen, ((d >> 5) & kMask) | kSixteen,
                       ((d >> 9) & kMask) | kSixteen};
    return __builtin_bit_cast(bf16x8_t, w);
}
// eight hidden values in the same order
__device__ __forceinline__ uint4 order_like_codes(const uint4 &v)
{
    return make_uint4(__builtin_amdgcn_perm(v.z, v.x, 0x05040100u), __builtin_amdgcn_perm(v.z, v.x, 0x07060302u),
                      __builtin_amdgcn_perm(v.w, v.y, 0x05040100u), __builtin_amdgcn_perm(v.w, v.y, 0x07060302u));
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

template <int GROUP, bool SCALE_F32>
struct Scales {
    static constexpr int kPerUnit = 128 / GROUP, kWords = SCALE_F32 ? kPerUnit : (kPerUnit + 1) / 2;
    uint32_t w[kWords];
    uint32_t zeros;
    __device__ __forceinline__ float scale(int g) const
    {
        if constexpr (SCALE_F32) return __uint_as_float(w[g]);
        else return __uint_as_float(g & 1 ? w[g / 2] & 0xFFFF0000u : w[g / 2] << 16);
    }
    __device__ __forceinline__ float zero(int g) const { return (float)(zeros >> (8 * g) & 0xFFu); }

    // the groups of one unit; `have` of them exist (the last unit of a row may be cut short)
    template <bool ZEROS>
    __device__ __forceinline__ void load(const void *s, const uint8_t *z, int64_t first, int have)
    {
        constexpr int kBytes = SCALE_F32 ? 4 : 2;
        const char *p = static_cast<const char *>(s) + first * kBytes;
        if (have >= kPerUnit) {
            if constexpr (kBytes * kPerUnit == 2) {
                w[0] = *reinterpret_cast<const uint16_t *>(p);
            } else if constexpr (kWords == 1) {
                typedef uint32_t word_t __attribute__((aligned(2)));
                w[0] = *reinterpret_cast<const word_t *>(p);
            } else {
                typedef uint32_t words_t __attribute__((ext_vector_type(kWords), aligned(kBytes)));
                const words_t v = *reinterpret_cast<const words_t *>(p);
#pragma unroll
                for (int i = 0; i < kWords; ++i) w[i] = v[i];
            }
            if constexpr (ZEROS) {
                if constexpr (kPerUnit == 1) {
                    zeros = z[first];
                } else if constexpr (kPerUnit == 2) {
                    typedef uint16_t half_t __attribute__((aligned(1)));
                    zeros = *reinterpret_cast<const half_t *>(z + first);
                } else {
                    typedef uint32_t word_t __attribute__((aligned(1)));
                    zeros = *reinterpret_cast<const word_t *>(z + first);
                }
            }
            return;
        }
        zeros = 0;
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
#pragma unroll
        for (int g = 0; g < kPerUnit; ++g)
            if (g < have) {
                if constexpr (SCALE_F32) w[g] = reinterpret_cast<const uint32_t *>(p)[g];
                else w[g / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[g] << (g & 1 ? 16 : 0);
                if constexpr (ZEROS) zeros |= (uint32_t)z[first + g] << (8 * g);
            }
    }
};

// MT: blocks of 16 tokens; R: blocks of 16 rows a wavefront.  The hidden values pass through LDS in chunks of 8 / MT units,
// two chunks at a time: one is read while the next arrives.
template <int MT, int R, int GROUP, bool ZEROS, bool SCALE_F32>
__global__ __launch_bounds__(kThreads) void w4_kernel(W4Args a)
{
    constexpr int UC = kWaves / MT, S = 128 / GROUP, BLOCKS = GROUP / 32;
    using Sc = Scales<GROUP, SCALE_F32>;
    __shared__ __align__(16) char xs[2][kWaves * 4 * kWave * 16];
    __shared__ __align__(16) float sums[2][kWaves * 4 * 16];
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int n16 = lane & 15, q = lane >> 4;
    const int units = (a.H + 127) / 128, chunks = (units + UC - 1) / UC;
    const int64_t t0 = (int64_t)blockIdx.y * (16 * MT), groups = a.H / GROUP;
    const int64_t n0 = (int64_t)blockIdx.x * (kWaves * R * 16) + wave * (R * 16);

    const char *codes[R];
    int64_t gbase[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t n = min(n0 + r * 16 + n16, a.V - 1);
        codes[r] = reinterpret_cast<const char *>(a.codes) + n * (a.H / 2);
        gbase[r] = n * groups;
    }
    // the unit and the 16 tokens of a chunk that this wavefront brings to LDS
    const int xu = wave / MT, xt = wave % MT;
    const int64_t token = t0 + xt * 16 + n16;
    const bool live = token < a.T;
    const char *xrow = reinterpret_cast<const char *>(a.x) + (live ? token : 0) * a.ldx * 2;

    uint4 xr[4];
    auto fetch_x = [&](int c) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int k = (c * UC + xu) * 128 + g * 32 + q * 8;
            xr[g] = make_uint4(0, 0, 0, 0);
            if (live && k < a.H) {
                const u32x4_half v = *reinterpret_cast<const u32x4_half *>(xrow + (int64_t)k * 2);
                xr[g] = make_uint4(v.x, v.y, v.z, v.w);
            }
        }
    };
    auto store_x = [&](int half) {
        float total = 0.0f;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            *reinterpret_cast<uint4 *>(xs[half] + (((xu * 4 + g) * MT + xt) * kWave + lane) * 16) = order_like_codes(xr[g]);
            float f[8], s;
            unpack<Bf16>(xr[g], f);
            s = ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
            s += __shfl_xor(s, 16, kWave);
            s += __shfl_xor(s, 32, kWave);
            total = g % BLOCKS == 0 ? s : total + s;
            // (the codes' excess: 16 + 8 without zero points)
            if (g % BLOCKS == BLOCKS - 1 && q == 0)
                sums[half][(xu * S + g / BLOCKS) * (16 * MT) + xt * 16 + n16] = ZEROS ? -total : -24.0f * total;
        }
    };

    uint4 wa[UC * R], wb[UC * R];
    Sc sa[UC * R], sb[UC * R];
    auto fetch_w = [&](int c, uint4 (&w)[UC * R], Sc (&s)[UC * R]) {
#pragma unroll
        for (int i = 0; i < UC; ++i) {
            const int u = c * UC + i;
            if (u < units) {
                const int left = (a.H - u * 128) / 32;  // blocks of this unit that exist
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const u32x4_t v = __builtin_nontemporal_load(
                        reinterpret_cast<const u32x4_t *>(codes[r] + (int64_t)u * 64 + min(q, left - 1) * 16));
                    w[i * R + r] = make_uint4(v.x, v.y, v.z, v.w);
                    s[i * R + r].template load<ZEROS>(a.scales, a.zeros, gbase[r] + (int64_t)u * S, left / BLOCKS);
                }
            }
        }
    };

    f32x4_t acc[R][MT];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[r][m] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

    auto multiply = [&](int c, int half, uint4 (&w)[UC * R], Sc (&s)[UC * R]) {
#pragma unroll
        for (int i = 0; i < UC; ++i) {
            if (c * UC + i >= units) break;
            uint32_t d[R][4];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const uint4 v = w[i * R + r];
                d[r][0] = v.x, d[r][1] = v.y, d[r][2] = v.z, d[r][3] = v.w;
                transpose_blocks(d[r]);
            }
            f32x4_t part[R][MT];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int gi = g / BLOCKS;
                if (g % BLOCKS == 0)
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        const f32x4_t e =
                            *reinterpret_cast<const f32x4_t *>(&sums[half][(i * S + gi) * (16 * MT) + m * 16 + q * 4]);
#pragma unroll
                        for (int r = 0; r < R; ++r) part[r][m] = ZEROS ? e * (16.0f + s[i * R + r].zero(gi)) : e;
                    }
                bf16x8_t wide[R];
#pragma unroll
                for (int r = 0; r < R; ++r) wide[r] = widen(d[r][g]);
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const bf16x8_t x = *reinterpret_cast<const bf16x8_t *>(xs[half] + (((i * 4 + g) * MT + m) * kWave + lane) * 16);
#pragma unroll
                    for (int r = 0; r < R; ++r)
                        part[r][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, wide[r], part[r][m], 0, 0, 0);
                }
                if (g % BLOCKS == BLOCKS - 1)
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int m = 0; m < MT; ++m) acc[r][m] += part[r][m] * s[i * R + r].scale(gi);
            }
        }
    };

    fetch_x(0);
    fetch_w(0, wa, sa);
    store_x(0);
    __syncthreads();
    for (int c = 0; c < chunks; c += 2) {
        if (c + 1 < chunks) {
            fetch_x(c + 1);
            fetch_w(c + 1, wb, sb);
        }
        multiply(c, 0, wa, sa);
        if (c + 1 >= chunks) break;
        store_x(1);
        __syncthreads();
        if (c + 2 < chunks) {
            fetch_x(c + 2);
            fetch_w(c + 2, wa, sa);
        }
        multiply(c + 1, 1, wb, sb);
        if (c + 2 >= chunks) break;
        store_x(0);
        __syncthreads();
    }

#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t n = n0 + r * 16 + n16;
        if (n >= a.V) continue;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t t = t0 + m * 16 + q * 4 + i;
                if (t < a.T) {
                    if (a.out_dt == A3PO_F32) static_cast<float *>(a.out)[t * a.ldo + n] = acc[r][m][i];
                    else store_elem<Bf16>(a.out, t * a.ldo + n, acc[r][m][i]);
                }
            }
    }
}

// ---- few tokens: hidden values resident -------------------------------------------------------------------------------
//
// All hidden values lie in LDS, in the order of the matrix instructions, for as long as the workgroup lives: one workgroup a
// compute unit, sixteen wavefronts.  A set of 16 x (16 / WK) rows is taken at a time: WK wavefronts share the 16 rows, a run of
// UPW units each, and add their sums through LDS.  A wavefront's weight is loaded NB sets ahead into registers (eight units or
// more in flight, 128 KiB a compute unit) and waits for nobody else's.

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

// a row's codes of UPW units in a row, with their scales and zero points
template <int UPW, int GROUP, bool ZEROS, bool SCALE_F32>
struct Run {
    static constexpr int kGroups = UPW * 128 / GROUP, kScaleBytes = kGroups * (SCALE_F32 ? 4 : 2);
    uint4 codes[UPW];
    uint32_t scales[(kScaleBytes + 3) / 4], zeros[ZEROS ? (kGroups + 3) / 4 : 1];
    __device__ __forceinline__ void load(const char *c, const char *s, const char *z)
    {
#pragma unroll
        for (int u = 0; u < UPW; ++u) {
            const u32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(c + u * 64));
            codes[u] = make_uint4(v.x, v.y, v.z, v.w);
        }
        load_run<kScaleBytes>(s, scales);
        if constexpr (ZEROS) load_run<kGroups>(z, zeros);
    }
    __device__ __forceinline__ float scale(int g) const
    {
        if constexpr (SCALE_F32) return __uint_as_float(scales[g]);
        else return __uint_as_float(g & 1 ? scales[g / 2] & 0xFFFF0000u : scales[g / 2] << 16);
    }
    __device__ __forceinline__ float zero(int g) const { return (float)(zeros[g / 4] >> (8 * (g % 4)) & 0xFFu); }
};

// a value in a scalar / vector register that the compiler knows nothing of (it would fold a constant into every instruction,
// of which an and-or can hold one only)
__device__ __forceinline__ uint32_t opaque_scalar(uint32_t v)
{
    asm("s_mov_b32 %0, %1" : "=s"(v) : "i"(0x00780078));
    return v;
}

__device__ __forceinline__ void meet()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(waitcnt_imm(kNoVmWait, 0));
    __builtin_amdgcn_s_barrier();  // (bare: the weight stays in flight)
    asm volatile("" ::: "memory");
}

template <int MT, int UPW, int NB, int GROUP, bool ZEROS, bool SCALE_F32>
__global__ __launch_bounds__(1024) void w4_resident_kernel(W4Args a, int wk_shift, int tp_shift, int sets)
{
    constexpr int S = 128 / GROUP, BLOCKS = GROUP / 32, kAll = 16;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int n16 = lane & 15, q = lane >> 4;
    const int WK = 1 << wk_shift, WR = kAll >> wk_shift, wk = wave & (WK - 1), wr = wave >> wk_shift;
    const int TP = MT > 1 ? 16 * MT : 1 << tp_shift;
    // (the last wavefronts' runs move down to end with the row; units that another one has as well count for nothing here)
    const int units = a.H >> 7, u0 = min(wk * UPW, units - UPW), skip = wk * UPW - u0;
    const int64_t groups = a.H / GROUP, row_bytes = a.H / 2;
    char *xs = lds;                                                             // [units][4][4][TP] 16 bytes
    float *sums = reinterpret_cast<float *>(lds + (size_t)a.H * TP * 2);        // [groups][TP]
    char *red = reinterpret_cast<char *>(sums + groups * TP);                   // [16 wavefronts][MT][64] 16 bytes

    // lane offsets from a set's first row (fewer than 16 rows in all: the last one again)
    const uint32_t row_lane = (uint32_t)min((int64_t)n16, a.V - 1);
    const uint32_t code_lane = row_lane * (uint32_t)row_bytes + q * 16, group_lane = row_lane * (uint32_t)groups;
    constexpr uint32_t kScale = SCALE_F32 ? 4 : 2;
    Run<UPW, GROUP, ZEROS, SCALE_F32> run[NB];
    // first row of this wavefront's block in a set; the last block moves up to end with the weight
    auto first_row = [&](int set) { return min(((int64_t)set * WR + wr) * 16, max(a.V - 16, (int64_t)0)); };
    // (no branch around the loads: at one the compiler waits for all that are in flight; sets beyond the last are the last)
    auto fetch = [&](int set, Run<UPW, GROUP, ZEROS, SCALE_F32> &to) {
        const int64_t row = first_row(min(set, sets - 1));
        const char *codes = reinterpret_cast<const char *>(a.codes) + row * row_bytes + u0 * 64;
        const int64_t group = row * groups + u0 * S;
        to.load(codes + code_lane, static_cast<const char *>(a.scales) + group * kScale + group_lane * kScale,
                ZEROS ? reinterpret_cast<const char *>(a.zeros) + group + group_lane : nullptr);
        __builtin_amdgcn_sched_barrier(0);  // (in this order: what is waited for first is issued first)
    };
#pragma unroll
    for (int b = 0; b < NB; ++b) fetch((int)blockIdx.x + b * (int)gridDim.x, run[b]);

    for (int p = threadIdx.x; p < units * 16 * TP; p += 1024) {
        const int token = p & (TP - 1), k8 = p / TP;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (token < a.T) {
            const u32x4_half h = *reinterpret_cast<const u32x4_half *>(static_cast<const char *>(a.x) + (token * a.ldx + k8 * 8) * 2);
            v = make_uint4(h.x, h.y, h.z, h.w);
        }
        // groups of a whole unit: the lanes of a block of codes keep it, and the quarter of the unit that they multiply is theirs
        const int at = GROUP == 128 ? (k8 & ~15) | (k8 & 3) << 2 | (k8 >> 2 & 3) : k8;
        *reinterpret_cast<uint4 *>(xs + ((size_t)at * TP + token) * 16) = order_like_codes(v);
    }
    meet();
    for (int p = threadIdx.x; p < (int)groups * TP; p += 1024) {
        const int token = p & (TP - 1), g = p / TP;
        float total = 0.0f;
#pragma unroll
        for (int k = 0; k < GROUP / 8; ++k) {
            float f[8];
            unpack<Bf16>(*reinterpret_cast<const uint4 *>(xs + ((size_t)(g * (GROUP / 8) + k) * TP + token) * 16), f);
            total += ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
        }
        sums[p] = ZEROS ? -total : -24.0f * total;  // (the codes' excess: 16 + 8 without zero points)
    }
    meet();

    const uint32_t mask = opaque_scalar(0);
    uint32_t sixteen;
    asm("v_mov_b32 %0, %1" : "=v"(sixteen) : "i"(0x41804180));
    auto widen_fast = [&](uint32_t d) {
        const u32x4_t v = {((d << 3) & mask) | sixteen, ((d >> 1) & mask) | sixteen, ((d >> 5) & mask) | sixteen,
                           ((d >> 9) & mask) | sixteen};
        return __builtin_bit_cast(bf16x8_t, v);
    };
    // (with fewer than 16 tokens the lanes of the others read these again; their products are not stored)
    const char *x_lane = xs + (q * TP + (n16 & (TP - 1))) * 16;
    const float *sum_lane = sums + ((q * 4) & (TP - 1));

    auto multiply = [&](const Run<UPW, GROUP, ZEROS, SCALE_F32> &from, f32x4_t (&acc)[MT]) {
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[m] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < UPW; ++u) {
            uint32_t d[4] = {from.codes[u].x, from.codes[u].y, from.codes[u].z, from.codes[u].w};
            if constexpr (GROUP < 128) transpose_blocks(d);
            const char *x = x_lane + (size_t)(u0 + u) * 16 * TP * 16;
            const float *sum = sum_lane + (u0 + u) * S * TP;
            f32x4_t part[MT];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int gi = g / BLOCKS;
                if (g % BLOCKS == 0)
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        part[m] = *reinterpret_cast<const f32x4_t *>(sum + gi * TP + m * 16);
                        if (ZEROS) part[m] *= 16.0f + from.zero(u * S + gi);
                    }
                const bf16x8_t wide = widen_fast(d[g]);
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    part[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        *reinterpret_cast<const bf16x8_t *>(x + ((size_t)g * 4 * TP + m * 16) * 16), wide, part[m], 0, 0, 0);
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
            if (row >= want && row < a.V) put_out(token, row, total);
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

template <int MT, int R, int GROUP, bool ZEROS, bool SCALE_F32>
hipError_t launch(const W4Args &a, hipStream_t s)
{
    constexpr int64_t kRows = kWaves * R * 16;
    const dim3 grid((unsigned)((a.V + kRows - 1) / kRows), (unsigned)((a.T + 16 * MT - 1) / (16 * MT)));
    w4_kernel<MT, R, GROUP, ZEROS, SCALE_F32><<<grid, dim3(kThreads), 0, s>>>(a);
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
    // registers of a unit in flight; as many units ahead as the 128 registers of sixteen wavefronts hold
    constexpr int kRegs = 4 + Scales<GROUP, SCALE_F32>::kWords + (ZEROS ? 1 : 0), kAhead = kRegs >= 8 ? 6 : kRegs == 7 && MT == 2 ? 8 : 9;
    if (p.units == 2) return launch_resident<MT, 2, kAhead / 2, GROUP, ZEROS, SCALE_F32>(a, p, s);
    if (p.units == 3) return launch_resident<MT, 3, kAhead / 3, GROUP, ZEROS, SCALE_F32>(a, p, s);
    if constexpr (kAhead >= 8) return launch_resident<MT, 4, kAhead / 4, GROUP, ZEROS, SCALE_F32>(a, p, s);
    return hipErrorInvalidValue;  // (w4_plan gives no such call four units)
}

template <int GROUP, bool ZEROS, bool SCALE_F32>
hipError_t launch_tokens(const W4Args &a, hipStream_t s)
{
    const GemmGrid chip = gemm_grid();
    const W4Plan p = w4_plan(a.T, a.H, a.V, a.group, SCALE_F32, (int64_t)chip.nxcd * chip.per_xcd);
    if (p.units && p.blocks16 == 1) return launch_units<1, GROUP, ZEROS, SCALE_F32>(a, p, s);
    if (p.units) return launch_units<2, GROUP, ZEROS, SCALE_F32>(a, p, s);
    if (a.T <= 16) return launch<1, 1, GROUP, ZEROS, SCALE_F32>(a, s);
    if (a.T <= 32) return launch<2, 1, GROUP, ZEROS, SCALE_F32>(a, s);
    return launch<4, 2, GROUP, ZEROS, SCALE_F32>(a, s);
}

template <int GROUP>
hipError_t launch_group(const W4Args &a, hipStream_t s)
{
    if (a.zeros) return a.scale_dt == A3PO_F32 ? launch_tokens<GROUP, true, true>(a, s) : launch_tokens<GROUP, true, false>(a, s);
    return a.scale_dt == A3PO_F32 ? launch_tokens<GROUP, false, true>(a, s) : launch_tokens<GROUP, false, false>(a, s);
}

}  // namespace

hipError_t launch_w4_linear(const W4Args &a, hipStream_t s)
{
    if (a.group == 32) return launch_group<32>(a, s);
    if (a.group == 64) return launch_group<64>(a, s);
    return launch_group<128>(a, s);
}

}  // namespace a3po
