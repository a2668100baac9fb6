// A weight in the layout that the 4-bit products read: 4-bit codes, a scale and maybe a zero point per group of a row.
//
//   zero points: scale = (max(hi, 0) - min(lo, 0)) / 15, zero = round(-min(lo, 0) / scale);  without: scale = max(hi / 7, -lo / 8),
//   zero = 8;  code = round(w / scale) + zero within [0, 15]
//
// A lane takes 8 elements of a group (16 bytes of bfloat16, 4 bytes of codes) and holds them while the group's 4, 8 or 16 lanes find its
// extremes: one read, one write, bound by memory.  151,936 x 1,536 bfloat16 in groups of 128: 112 us, 5.3 TB/s; 32,001 x 4,096 fp32 in
// groups of 32 with zero points 124 us, 4.9 TB/s.
#include "a3po_common.h"
#include "a3po_launch.h"

namespace a3po {
namespace {

constexpr int kThreads = 256;

template <typename DT, bool SCALE_F32, bool ZEROS, int LANES>
__global__ __launch_bounds__(kThreads) void w4_quantize_kernel(W4QuantizeArgs a)
{
    const int64_t per_row = a.H / 8, all = a.N * per_row;  // lanes' pieces of 8 elements; a group's are LANES in a row
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < all; i += (int64_t)gridDim.x * kThreads) {
        const int64_t row = i / per_row, at = i - row * per_row;
        const char *p = reinterpret_cast<const char *>(a.w) + (row * a.ld + at * 8) * DT::kBytes;
        float w[8];
#pragma unroll
        for (int k = 0; k < 8; k += DT::kPerVec) unpack<DT>(row_load<true>(p + k * DT::kBytes), w + k);
        float hi = w[0], lo = w[0];
#pragma unroll
        for (int k = 1; k < 8; ++k) hi = fmaxf(hi, w[k]), lo = fminf(lo, w[k]);
#pragma unroll
        for (int off = 1; off < LANES; off <<= 1) hi = fmaxf(hi, __shfl_xor(hi, off, kWave)), lo = fminf(lo, __shfl_xor(lo, off, kWave));
        if constexpr (ZEROS) hi = fmaxf(hi, 0.0f), lo = fminf(lo, 0.0f);
        float scale = ZEROS ? (hi - lo) * (1.0f / 15.0f) : fmaxf(hi * (1.0f / 7.0f), lo * -0.125f);
        if constexpr (ZEROS)  // (a range beyond fp32's largest number)
            if (scale > 3.402823466e38f) scale = hi * (1.0f / 15.0f) - lo * (1.0f / 15.0f);
        uint32_t scale16 = 0;
        if constexpr (!SCALE_F32) scale16 = pack_bf16x2(scale, 0.0f) & 0xFFFFu, scale = bf16_bits_to_float(scale16);
        const float inverse = scale >= 1.17549435e-38f ? 1.0f / scale : 0.0f;
        const float zero = ZEROS ? fminf(fmaxf(rintf(-lo * inverse), 0.0f), 15.0f) : 8.0f;
        uint32_t codes = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            codes |= (uint32_t)fminf(fmaxf(rintf(w[k] * inverse) + zero, 0.0f), 15.0f) << (4 * k);
        reinterpret_cast<uint32_t *>(a.codes)[i] = codes;
        if ((threadIdx.x & (LANES - 1)) == 0) {
            const int64_t g = i / LANES;
            if constexpr (SCALE_F32) reinterpret_cast<float *>(a.scales)[g] = scale;
            else reinterpret_cast<uint16_t *>(a.scales)[g] = (uint16_t)scale16;
            if constexpr (ZEROS) a.zeros[g] = (uint8_t)zero;
        }
    }
}

template <typename DT, bool SCALE_F32, bool ZEROS>
void launch(const W4QuantizeArgs &a, hipStream_t s)
{
    const int64_t need = (a.N * (a.H / 8) + kThreads - 1) / kThreads;
    const int grid = (int)(need < 256 * 64 ? need : 256 * 64);
    if (a.group == 32) w4_quantize_kernel<DT, SCALE_F32, ZEROS, 4><<<grid, kThreads, 0, s>>>(a);
    else if (a.group == 64) w4_quantize_kernel<DT, SCALE_F32, ZEROS, 8><<<grid, kThreads, 0, s>>>(a);
    else w4_quantize_kernel<DT, SCALE_F32, ZEROS, 16><<<grid, kThreads, 0, s>>>(a);
}

}  // namespace

hipError_t launch_w4_quantize(const W4QuantizeArgs &a, hipStream_t s)
{
    const bool f = a.scale_dt == A3PO_F32, z = a.zeros != nullptr;
    if (a.dt == A3PO_F32) {
        if (f) z ? launch<F32, true, true>(a, s) : launch<F32, true, false>(a, s);
        else z ? launch<F32, false, true>(a, s) : launch<F32, false, false>(a, s);
    } else {
        if (f) z ? launch<Bf16, true, true>(a, s) : launch<Bf16, true, false>(a, s);
        else z ? launch<Bf16, false, true>(a, s) : launch<Bf16, false, false>(a, s);
    }
    return hipGetLastError();
}

}  // namespace a3po
