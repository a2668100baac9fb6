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
            } else {
                typedef uint32_t words_t __attribute__((ext_vector_type(kWords), aligned(kBytes)));
                const words_t v = *reinterpret_cast<const words_t *>(p);
                if constexpr (kWords == 1) w[0] = v[0];
                else
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

template <int MT, int R, int GROUP, bool ZEROS, bool SCALE_F32>
hipError_t launch(const W4Args &a, hipStream_t s)
{
    constexpr int64_t kRows = kWaves * R * 16;
    const dim3 grid((unsigned)((a.V + kRows - 1) / kRows), (unsigned)((a.T + 16 * MT - 1) / (16 * MT)));
    w4_kernel<MT, R, GROUP, ZEROS, SCALE_F32><<<grid, dim3(kThreads), 0, s>>>(a);
    return hipGetLastError();
}

template <int GROUP, bool ZEROS, bool SCALE_F32>
hipError_t launch_tokens(const W4Args &a, hipStream_t s)
{
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
