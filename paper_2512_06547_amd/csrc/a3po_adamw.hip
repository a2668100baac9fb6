// A step of AdamW over many tensors, with states in 32 bits or in 8, and the norm of all gradients that clips it.
//
//   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
//   p = p (1 - lr decay) - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
//
// States in 8 bits: blocks of 32 elements share a power of two, m as float8 e4m3 (the largest of a block between 2^7 and 2^8), v
// as e5m2 (between 2^14 and 2^15: 31 powers of two below the largest, twice m's range as it holds squares).  m is rounded to
// nearest: a step takes at least a tenth of it or adds to it.  v loses a thousandth a step where half of its last bit is a
// sixteenth: to nearest it would never fall, so it goes up or down by chance with itself as the mean, but never to zero from
// above, which would leave m divided by eps alone.
//
// Memory bounds it: a thread reads 8 elements of everything, 16 bytes at a time, past the caches, and writes them back; 2,048 a
// workgroup, as many workgroups as there are chunks (no element is read twice, so nothing is gained by fewer).  151,936 x 1,536
// fp32 weights with bfloat16 gradients and copies: states in 32 bits 28 bytes an element, 1,270 us, 5.1 TB/s; in 8 bits 16.1 bytes, 707 us,
// 5.3 TB/s (495 vector instructions a wavefront, 57 % of the cycles).  The gradients' norm reads them once more, 83 us: the step needs
// it before its first element.  With the step's number on the device each thread computes the two powers of beta in 64 bits for itself: the
// same weights 8 us more, with 8-bit states 49.
#include "a3po_common.h"
#include "a3po_launch.h"

namespace a3po {
namespace {

constexpr int kThreads = 256, kEach = 8, kChunk = kThreads * kEach;

// Addresses have 48 bits: the upper 16 of two share a word, and the eighth 16 say how many elements the last chunk has.  (80 tensors a
// launch, 40 with the fields as they are: 300 odd tensors of 5 * 10^7 bfloat16 elements and 8-bit states take 129 us, and took 177)
struct AdamTensor {
    enum { kParam, kGrad, kM, kV, kCopy, kMScale, kVScale, kPointers };
    uint32_t low[kPointers], high[(kPointers + 1) / 2];
    __device__ __forceinline__ uint32_t upper(int i) const { return high[i / 2] >> (16 * (i & 1)) & 0xFFFFu; }
    template <typename T = char>
    __device__ __forceinline__ T *at(int i) const
    {
        typedef T __attribute__((address_space(1))) global_t;  // (flat loads would count as LDS's too)
        return (T *)reinterpret_cast<global_t *>((uint64_t)upper(i) << 32 | low[i]);
    }
};
struct AdamArgs {
    AdamTensor tensor[kAdamTensors];
    uint32_t first[kAdamTensors + 1];  // chunk of each tensor's beginning
    int count;
    uint32_t seed, number;  // number: of the first tensor
    float beta1, rest1, beta2, rest2, eps, decay, size, root;  // rest: 1 - beta; size: lr / (1 - beta1^t); root: 1 / sqrt(1 - beta2^t)
    float max_norm;
    const float *norm, *lr_dev;
    const int64_t *step_dev;
    double lr, weight_decay, dbeta1, dbeta2;
    int64_t step;
};
static_assert(sizeof(AdamArgs) <= 4096, "launch arguments");

// 32 bits of chance for every whole number: two multiplications between shifted sums without carry.  Shifts and factors are those of a
// published function, the last step of Austin Appleby's MurmurHash3 for 32 bits (public domain).
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x)
{
    x ^= x >> 16;
    x *= 0x85EBCA6Bu;
    x ^= x >> 13;
    x *= 0xC2B2AE35u;
    return x ^ x >> 16;
}

typedef u32x4_t u32x4_byte_t __attribute__((aligned(1)));
typedef uint32_t u32x2_byte_t __attribute__((ext_vector_type(2), aligned(1)));

// kEach elements at p, or the first `left` of them and zeros behind
template <typename DT>
__device__ __forceinline__ void load8(const void *p, int64_t at, int left, float *f)
{
    const char *q = reinterpret_cast<const char *>(p) + at * DT::kBytes;
    if (left >= kEach) {
#pragma unroll
        for (int k = 0; k < kEach; k += DT::kPerVec) unpack<DT>(row_load<true>(q + k * DT::kBytes), f + k);
    } else {
#pragma unroll
        for (int k = 0; k < kEach; ++k) f[k] = k < left ? load_elem<DT>(q, k) : 0.0f;
    }
}
template <typename DT>
__device__ __forceinline__ void store8(void *p, int64_t at, int left, const float *f)
{
    char *q = reinterpret_cast<char *>(p) + at * DT::kBytes;
    if (left >= kEach) {
#pragma unroll
        for (int k = 0; k < kEach; k += DT::kPerVec) {
            const uint4 v = pack<DT>(f + k);
            const u32x4_t t = {v.x, v.y, v.z, v.w};
            __builtin_nontemporal_store(t, reinterpret_cast<u32x4_elem_t *>(q + k * DT::kBytes));
        }
    } else {
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            if (k < left) store_elem<DT>(q, k, f[k]);
    }
}
__device__ __forceinline__ void load_bytes(const void *p, int64_t at, int left, uint32_t (&w)[2])
{
    const uint8_t *q = reinterpret_cast<const uint8_t *>(p) + at;
    if (left >= kEach) {
        const u32x2_byte_t t = *reinterpret_cast<const u32x2_byte_t *>(q);
        w[0] = t.x, w[1] = t.y;
    } else {
        w[0] = w[1] = 0;
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            if (k < left) w[k / 4] |= (uint32_t)q[k] << (8 * (k & 3));
    }
}
__device__ __forceinline__ void store_bytes(void *p, int64_t at, int left, const uint32_t (&w)[2])
{
    uint8_t *q = reinterpret_cast<uint8_t *>(p) + at;
    if (left >= kEach) {
        const u32x2_byte_t t = {w[0], w[1]};
        *reinterpret_cast<u32x2_byte_t *>(q) = t;
    } else {
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            if (k < left) q[k] = (uint8_t)(w[k / 4] >> (8 * (k & 3)));
    }
}

// the largest bit pattern of the four lanes that share a block
__device__ __forceinline__ uint32_t block_max(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));
    return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));
}

// the block's exponent byte for its largest magnitude to have the exponent `top`, and the factor that takes values there
__device__ __forceinline__ uint32_t block_exponent(uint32_t largest, int top, float &up, bool &finite)
{
    const int e = (int)(largest >> 23), scale = max(e - top, 1);
    finite = e < 255;
    up = __uint_as_float((uint32_t)(254 - scale) << 23);
    return finite ? (uint32_t)scale : 255u;
}

__device__ __forceinline__ void decode_m(const uint32_t (&w)[2], uint32_t scale, float *f)
{
    const float unit = __uint_as_float(scale << 23);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
        f[4 * k] = a.x * unit, f[4 * k + 1] = a.y * unit, f[4 * k + 2] = b.x * unit, f[4 * k + 3] = b.y * unit;
    }
}
__device__ __forceinline__ void decode_v(const uint32_t (&w)[2], uint32_t scale, float *f)
{
    const float unit = __uint_as_float(scale << 23);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_bf8((int)w[k], false), b = __builtin_amdgcn_cvt_pk_f32_bf8((int)w[k], true);
        f[4 * k] = a.x * unit, f[4 * k + 1] = a.y * unit, f[4 * k + 2] = b.x * unit, f[4 * k + 3] = b.y * unit;
    }
}
__device__ __forceinline__ uint32_t encode_m(const float *f, uint32_t (&w)[2])
{
    uint32_t largest = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) largest = max(largest, __float_as_uint(f[k]) & 0x7FFFFFFFu);
    float up;
    bool finite;
    const uint32_t scale = block_exponent(block_max(largest), 7, up, finite);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        int t = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * k] * up, f[4 * k + 1] * up, 0, false);
        t = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * k + 2] * up, f[4 * k + 3] * up, t, true);
        w[k] = finite ? (uint32_t)t : 0x7F7F7F7Fu;
    }
    return scale;
}
// v >= 0: up or down by the low 21 random bits, which are what e5m2 leaves of a mantissa
__device__ __forceinline__ uint32_t encode_v(const float *f, const uint32_t *chance, uint32_t (&w)[2])
{
    uint32_t largest = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) largest = max(largest, __float_as_uint(f[k]));
    float up;
    bool finite;
    const uint32_t scale = block_exponent(block_max(largest), 14, up, finite);
    w[0] = w[1] = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const float x = f[k] * up;
        const uint32_t r = chance[k] & 0x1FFFFFu;
        uint32_t code = ((__float_as_uint(x) + r) >> 21) - 448u;
        // below 2^-14 the numbers are multiples of 2^-16
        if (x < 6.103515625e-5f) code = (uint32_t)fmaf(x, 65536.0f, (float)r * 4.76837158203125e-7f);
        if (x > 0.0f) code = max(code, 1u);
        w[k / 4] |= (code & 0xFFu) << (8 * (k & 3));
    }
    if (!finite) w[0] = w[1] = 0x7F7F7F7Fu;
    return scale;
}

template <typename PT, typename GT, bool BYTES>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const AdamArgs a)
{
    float factor = 1.0f, decay = a.decay, size = a.size, root = a.root;
    if (a.norm) {
        const float norm = *a.norm;
        if (!(fabsf(norm) < __builtin_huge_valf())) return;
        factor = fminf(a.max_norm / (norm + 1e-6f), 1.0f);
    }
    if (a.lr_dev || a.step_dev) {
        const double lr = a.lr_dev ? (double)*a.lr_dev : a.lr, step = (double)(a.step_dev ? *a.step_dev : a.step);
        decay = (float)(1.0 - lr * a.weight_decay);
        size = (float)(lr / (1.0 - pow(a.dbeta1, step)));
        root = (float)(1.0 / sqrt(1.0 - pow(a.dbeta2, step)));
    }
    // (a replayed graph's seed is always the one it was captured with)
    const uint32_t salt = a.step_dev ? mix((uint32_t)*a.step_dev) : 0u;
    const uint32_t chunks = a.first[a.count];
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        int k = 0;
        for (int step = 64; step; step >>= 1)
            if (k + step < a.count && a.first[k + step] <= c) k += step;
        const AdamTensor t = a.tensor[k];
        const int64_t at = (int64_t)(c - a.first[k]) * kChunk + (int)threadIdx.x * kEach;
        const int here = c + 1 == a.first[k + 1] ? (int)t.upper(AdamTensor::kPointers) : kChunk;
        const int left = max(0, min(here - (int)threadIdx.x * kEach, kEach));
        float p[kEach], g[kEach], m[kEach], v[kEach];
        uint32_t wm[2], wv[2];
        load8<PT>(t.at(AdamTensor::kParam), at, left, p);
        load8<GT>(t.at(AdamTensor::kGrad), at, left, g);
        if constexpr (BYTES) {
            load_bytes(t.at(AdamTensor::kM), at, left, wm);
            load_bytes(t.at(AdamTensor::kV), at, left, wv);
            decode_m(wm, left > 0 ? t.at<uint8_t>(AdamTensor::kMScale)[at / 32] : 0u, m);
            decode_v(wv, left > 0 ? t.at<uint8_t>(AdamTensor::kVScale)[at / 32] : 0u, v);
        } else {
            load8<F32>(t.at(AdamTensor::kM), at, left, m);
            load8<F32>(t.at(AdamTensor::kV), at, left, v);
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            // (each product and sum of the states is rounded, so that they are what the formulas give in fp32 anywhere: with bfloat16 gradients and
            // beta1 = 0.9 a new mean often is a tie of two bytes, which a product that enters its sum unrounded would decide otherwise)
#pragma clang fp contract(off)
            const float x = g[i] * factor;
            m[i] = a.beta1 * m[i] + a.rest1 * x;
            v[i] = a.beta2 * v[i] + a.rest2 * x * x;
            // (the root's instruction takes numbers below 2^-126 for 0)
            const bool tiny = v[i] < 0x1p-96f;
            const float below = fmaf(__builtin_amdgcn_sqrtf(tiny ? v[i] * 0x1p64f : v[i]), tiny ? root * 0x1p-32f : root, a.eps);
            // (where there has been no gradient yet and eps is 0, the mean over its root is 0 over 0: no update)
            p[i] = fmaf(p[i], decay, m[i] == 0.0f ? 0.0f : -size * (m[i] * __builtin_amdgcn_rcpf(below)));
        }
        // (a bfloat16 weight is rounded by the upper 16 bits, exp_avg_sq by the lower 21: an element that has both shares five of them)
        uint32_t chance[kEach];
        if constexpr (BYTES || PT::kBytes == 2) {
            const uint32_t key = mix(a.seed + 0x9E3779B9u * (a.number + (uint32_t)k + 1u)) ^ salt ^ (uint32_t)(at >> 32) * 0x9E3779B9u;
#pragma unroll
            for (int i = 0; i < kEach; ++i) chance[i] = mix(((uint32_t)at + i) ^ key);
        }
        if constexpr (PT::kBytes == 2) {
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (fabsf(p[i]) < __builtin_huge_valf()) p[i] = __uint_as_float((__float_as_uint(p[i]) + (chance[i] >> 16)) & 0xFFFF0000u);
        }
        store8<PT>(t.at(AdamTensor::kParam), at, left, p);
        if (char *copy = t.at(AdamTensor::kCopy)) store8<Bf16>(copy, at, left, p);
        if constexpr (BYTES) {
            const uint32_t sm = encode_m(m, wm), sv = encode_v(v, chance, wv);
            store_bytes(t.at(AdamTensor::kM), at, left, wm);
            store_bytes(t.at(AdamTensor::kV), at, left, wv);
            if (left > 0 && (threadIdx.x & 3) == 0) t.at<uint8_t>(AdamTensor::kMScale)[at / 32] = (uint8_t)sm, t.at<uint8_t>(AdamTensor::kVScale)[at / 32] = (uint8_t)sv;
        } else {
            store8<F32>(t.at(AdamTensor::kM), at, left, m);
            store8<F32>(t.at(AdamTensor::kV), at, left, v);
        }
    }
}

// ---- norm of all gradients -------------------------------------------------------------------------------------------

constexpr int kNormChunk = kThreads * 32;

struct SquaresArgs {
    const void *grad[kNormTensors];
    int64_t n[kNormTensors];
    int count;
};
static_assert(sizeof(SquaresArgs) <= 4096, "launch arguments");

__device__ __forceinline__ double block_sum(double v, double *waves)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, n = blockDim.x / kWave;
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
    if (lane == 0) waves[wave] = v;
    __syncthreads();
    double sum = 0.0;
    for (int w = 0; w < n; ++w) sum += waves[w];
    return sum;
}

// A workgroup takes every gridDim-th chunk of all tensors' elements, counted through; squares are added in 64 bits, by tensor, place and
// then workgroup, so in one order always.  233 million bfloat16 elements 83 us, 5.6 TB/s.
template <typename GT>
__global__ __launch_bounds__(kThreads) void grad_squares_kernel(const SquaresArgs a, double *partial)
{
    __shared__ double waves[kThreads / kWave];
    double sum = 0.0;
    int64_t before = 0;  // chunks of the tensors so far
    int64_t c = blockIdx.x;
    for (int k = 0; k < a.count; ++k) {
        const int64_t n = a.n[k], chunks = (n + kNormChunk - 1) / kNormChunk;
        for (; c < before + chunks; c += gridDim.x) {
            const int64_t at = (c - before) * kNormChunk + (int)threadIdx.x * kEach;
#pragma unroll
            for (int j = 0; j < kNormChunk / kChunk; ++j) {
                const int64_t e = at + j * kChunk;
                float g[kEach];
                load8<GT>(a.grad[k], e, (int)max((int64_t)0, min(n - e, (int64_t)kEach)), g);
#pragma unroll
                for (int i = 0; i < kEach; ++i) sum = fma((double)g[i], (double)g[i], sum);
            }
        }
        before += chunks;
    }
    sum = block_sum(sum, waves);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__global__ __launch_bounds__(1024) void grad_norm_kernel(const double *partial, int64_t count, float scale, float *norm)
{
    __shared__ double waves[1024 / kWave];
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < count; i += 1024) sum += partial[i];
    sum = block_sum(sum, waves);
    if (threadIdx.x == 0) *norm = (float)(fabs((double)scale) * sqrt(sum));
}

template <typename PT, typename GT>
void launch_step(const AdamArgs &a, int grid, bool bytes, hipStream_t s)
{
    if (bytes) adamw_kernel<PT, GT, true><<<grid, kThreads, 0, s>>>(a);
    else adamw_kernel<PT, GT, false><<<grid, kThreads, 0, s>>>(a);
}

}  // namespace

hipError_t launch_adamw(const a3po_adamw_tensor *tensors, int64_t count, int param_dt, int grad_dt, int state_format,
                        const a3po_adamw_options &o, hipStream_t s)
{
    AdamArgs a = {};
    a.beta1 = (float)o.beta1, a.rest1 = (float)(1.0 - o.beta1), a.beta2 = (float)o.beta2, a.rest2 = (float)(1.0 - o.beta2);
    a.eps = (float)o.eps;
    a.max_norm = (float)o.max_norm;
    a.norm = o.norm, a.lr_dev = o.lr_dev, a.step_dev = o.step_dev;
    a.lr = o.lr, a.weight_decay = o.weight_decay, a.dbeta1 = o.beta1, a.dbeta2 = o.beta2, a.step = o.step;
    a.decay = (float)(1.0 - o.lr * o.weight_decay);
    a.size = (float)(o.lr / (1.0 - std::pow(o.beta1, (double)o.step)));
    a.root = (float)(1.0 / std::sqrt(1.0 - std::pow(o.beta2, (double)o.step)));
    const bool bytes = state_format == A3PO_STATE_8BIT;
    a.seed = o.seed;
    for (int64_t i = 0; i < count;) {
        int k = 0;
        a.number = (uint32_t)i;
        for (; i < count && k < kAdamTensors; ++i, ++k) {  // (an empty tensor has no chunks)
            const a3po_adamw_tensor &t = tensors[i];
            const int64_t chunks = (t.n + kChunk - 1) / kChunk;
            if (a.first[k] + chunks > 0x7FFFFFFF) break;
            const void *const fields[] = {t.param, t.grad, t.exp_avg, t.exp_avg_sq, t.copy, t.exp_avg_scale, t.exp_avg_sq_scale};
            AdamTensor &to = a.tensor[k];
            to = {};
            for (int f = 0; f < AdamTensor::kPointers; ++f) {
                const uint64_t at = reinterpret_cast<uint64_t>(fields[f]);
                if (at >> 48) return hipErrorInvalidValue;
                to.low[f] = (uint32_t)at, to.high[f / 2] |= (uint32_t)(at >> 32) << (16 * (f & 1));
            }
            to.high[AdamTensor::kPointers / 2] |= (uint32_t)(t.n - (chunks - 1) * kChunk) << (16 * (AdamTensor::kPointers & 1));
            a.first[k + 1] = a.first[k] + (uint32_t)chunks;
        }
        a.count = k;
        if (a.first[k] == 0) continue;
        const int grid = (int)(a.first[k] < (1u << 22) ? a.first[k] : 1u << 22);
        if (param_dt == A3PO_F32) grad_dt == A3PO_F32 ? launch_step<F32, F32>(a, grid, bytes, s) : launch_step<F32, Bf16>(a, grid, bytes, s);
        else grad_dt == A3PO_F32 ? launch_step<Bf16, F32>(a, grid, bytes, s) : launch_step<Bf16, Bf16>(a, grid, bytes, s);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_grad_norm(const void *const *grads, const int64_t *sizes, int64_t count, int dt, float scale, float *norm,
                            void *workspace, hipStream_t s)
{
    double *partial = static_cast<double *>(workspace);
    int64_t partials = 0;
    SquaresArgs a = {};
    for (int64_t i = 0; i < count;) {
        int k = 0;
        int64_t chunks = 0;
        for (; i < count && k < kNormTensors; ++i) {
            if (sizes[i] == 0) continue;
            a.grad[k] = grads[i], a.n[k] = sizes[i];
            chunks += (sizes[i] + kNormChunk - 1) / kNormChunk;
            ++k;
        }
        if (k == 0) break;
        a.count = k;
        const int grid = (int)(chunks < kNormBlocks ? chunks : kNormBlocks);
        if (dt == A3PO_F32) grad_squares_kernel<F32><<<grid, kThreads, 0, s>>>(a, partial + partials);
        else grad_squares_kernel<Bf16><<<grid, kThreads, 0, s>>>(a, partial + partials);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        partials += grid;
    }
    grad_norm_kernel<<<1, 1024, 0, s>>>(partial, partials, scale, norm);
    return hipGetLastError();
}

}  // namespace a3po
