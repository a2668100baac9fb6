// Layer norm and its root-mean-square form over rows of hidden states, forward and backward.
//
//   c = x - mean (mean = 0 in the root-mean-square form),  rstd = 1 / sqrt(mean(c^2) + eps),  xhat = c rstd
//   y = xhat w + b
//   dx = rstd (g - mean(g) - xhat mean(g xhat)),  g = dy w   (without mean(g) in the root-mean-square form)
//   dw = sum over rows of dy xhat,  db = sum over rows of dy
//
// Both passes keep each row in registers and read it once (the gradient of few rows a second time, for the sums over rows);
// statistics, products and sums are fp32, and every output is rounded once.  The variance is the mean of (x - mean)^2, taken from
// the registers after the mean is known: the difference of two sums loses all digits of rows whose mean is large against their
// spread.
// The kernels are bound by memory where there are rows enough: the gradient of 65,536 x 4,096 bfloat16 moves 1.61 GB in 280 us
// (5.8 TB/s), the forward pass of 10,240 x 2,049 fp32 to bfloat16 126 MB in 25.  Fewer rows are a chain of latencies, a load, two
// reductions and a store: 64 x 1,536 forward 3.5 us, 1,000 x 1,536 fp32 backward 10.5.
#include <type_traits>

#include "a3po_common.h"
#include "a3po_launch.h"

namespace a3po {
namespace {

// LANES lanes share a row: each holds NV vectors of EPV elements (16 bytes of x), vector i at (i LANES + lane) EPV, and
// one element of what is left of the row behind the last whole vector.  Rows may start at any element.
template <typename XT>
constexpr int kVec = 16 / XT::kBytes;

// EPV consecutive elements of type DT, widened
template <typename DT, int EPV, bool STREAM = false>
__device__ __forceinline__ void load_vec(const char *p, float *f)
{
    constexpr int kWords = EPV * DT::kBytes / 4;
    typedef uint32_t words_t __attribute__((ext_vector_type(kWords < 4 ? kWords : 4), aligned(DT::kBytes)));
    constexpr int kPer = kWords < 4 ? kWords : 4;
#pragma unroll
    for (int k = 0; k < kWords; k += kPer) {
        words_t w;
        if constexpr (STREAM) w = __builtin_nontemporal_load(reinterpret_cast<const words_t *>(p + 4 * k));
        else w = *reinterpret_cast<const words_t *>(p + 4 * k);
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            if constexpr (DT::kBytes == 4) {
                f[k + j] = __uint_as_float(w[j]);
            } else {
                f[2 * (k + j)] = __uint_as_float(w[j] << 16);
                f[2 * (k + j) + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
            }
        }
    }
}

template <typename DT, int EPV, bool STREAM = false>
__device__ __forceinline__ void store_vec(char *p, const float *f)
{
    constexpr int kWords = EPV * DT::kBytes / 4;
    constexpr int kPer = kWords < 4 ? kWords : 4;
    typedef uint32_t words_t __attribute__((ext_vector_type(kPer), aligned(DT::kBytes)));
#pragma unroll
    for (int k = 0; k < kWords; k += kPer) {
        words_t w;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            if constexpr (DT::kBytes == 4) w[j] = __float_as_uint(f[k + j]);
            else w[j] = pack_bf16x2(f[2 * (k + j)], f[2 * (k + j) + 1]);
        }
        if constexpr (STREAM) __builtin_nontemporal_store(w, reinterpret_cast<words_t *>(p + 4 * k));
        else *reinterpret_cast<words_t *>(p + 4 * k) = w;
    }
}

// a weight or bias vector, whose type is the call's (one value for the whole grid); `none` where there is no array
template <int EPV>
__device__ __forceinline__ void load_param(const void *w, bool f32, int64_t e, float none, float *f)
{
    if (!w) {
#pragma unroll
        for (int k = 0; k < EPV; ++k) f[k] = none;
    } else if (f32) {
        load_vec<F32, EPV>(static_cast<const char *>(w) + 4 * e, f);
    } else {
        load_vec<Bf16, EPV>(static_cast<const char *>(w) + 2 * e, f);
    }
}
__device__ __forceinline__ float load_param(const void *w, bool f32, int64_t e, float none)
{
    if (!w) return none;
    return f32 ? load_elem<F32>(w, e) : load_elem<Bf16>(w, e);
}

// Sums over the LANES lanes of a row; every lane gets them.  With several wavefronts a row they pass through `red`,
// which alternates between two halves from row to row, so that one barrier a sum is enough.
template <int LANES, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float (*red)[2 * (LANES / kWave)], int &phase)
{
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int off = kWave / 2; off > 0; off >>= 1) v[n] += __shfl_xor(v[n], off, kWave);
    if constexpr (LANES > kWave) {
        constexpr int kWaves = LANES / kWave;
        const int wave = threadIdx.x / kWave;
        if ((threadIdx.x & (kWave - 1)) == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) red[phase][N * wave + n] = v[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
#pragma unroll
            for (int n = 0; n < N; ++n) v[n] += red[phase][N * w + n];
        phase ^= 1;
    }
}

// Vectors beyond the row's last whole one read that one again and count for nothing: with a branch around each vector's load
// its use waits for it alone, one after the other.  (Rows shorter than a vector have none.)
template <typename XT, typename YT, int LANES, int NV, bool CENTER>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void norm_fwd_kernel(NormArgs a)
{
    constexpr int EPV = kVec<XT>, kRows = LANES >= 256 ? 1 : 256 / LANES;
    __shared__ float red[2][2 * (LANES / kWave)];
    int phase = 0;
    const int lane = threadIdx.x % LANES, full = a.H / EPV, rest = a.H - full * EPV, e_last = full * EPV + lane;
    const float inv_h = 1.0f / (float)a.H;
    const bool last = lane < rest;
    float w[NV][EPV], b[CENTER ? NV : 1][EPV], w_last = 0.0f, b_last = 0.0f;
    if (full)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t e = (int64_t)min(i * LANES + lane, full - 1) * EPV;
            load_param<EPV>(a.weight, a.param_f32, e, 1.0f, w[i]);
            if constexpr (CENTER) load_param<EPV>(a.bias, a.param_f32, e, 0.0f, b[i]);
        }
    if (last) {
        w_last = load_param(a.weight, a.param_f32, e_last, 1.0f);
        b_last = load_param(a.bias, a.param_f32, e_last, 0.0f);
    }
    const int64_t stride = (int64_t)gridDim.x * kRows;
    for (int64_t t = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES; t < a.T; t += stride) {
        const char *row = static_cast<const char *>(a.x) + t * a.ldx * XT::kBytes;
        char *out = static_cast<char *>(a.y) + t * a.ldy * YT::kBytes;
        float f[NV][EPV], extra = 0.0f;
        if (full)
#pragma unroll
            for (int i = 0; i < NV; ++i) load_vec<XT, EPV>(row + min(i * LANES + lane, full - 1) * EPV * XT::kBytes, f[i]);
        if (last) extra = load_elem<XT>(row, e_last);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < EPV; ++k) f[i][k] = i * LANES + lane < full ? f[i][k] : 0.0f;
        float mean = 0.0f;
        if constexpr (CENTER) {
            float sum[1] = {extra};
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < EPV; ++k) sum[0] += f[i][k];
            row_sum<LANES, 1>(sum, red, phase);
            mean = sum[0] / (float)a.H;  // (divided: rows of equal values have that mean exactly)
        }
        float sq[1] = {last ? (extra - mean) * (extra - mean) : 0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool on = i * LANES + lane < full;
#pragma unroll
            for (int k = 0; k < EPV; ++k) {
                if constexpr (CENTER) f[i][k] = on ? f[i][k] - mean : 0.0f;
                sq[0] = fmaf(f[i][k], f[i][k], sq[0]);
            }
        }
        row_sum<LANES, 1>(sq, red, phase);
        const float rstd = 1.0f / sqrtf(fmaf(sq[0], inv_h, a.eps));
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * LANES + lane;
            if (v < full) {
#pragma unroll
                for (int k = 0; k < EPV; ++k) f[i][k] = fmaf(f[i][k] * rstd, w[i][k], CENTER ? b[i][k] : 0.0f);
                store_vec<YT, EPV>(out + v * EPV * YT::kBytes, f[i]);
            }
        }
        if (last) store_elem<YT>(out, e_last, fmaf((extra - mean) * rstd, w_last, b_last));
        if (lane == 0) {
            if (a.mean) a.mean[t] = mean;
            if (a.rstd) a.rstd[t] = rstd;
        }
    }
}

// The sums over rows of 4 vectors of columns, straight from x and dy (mean and rstd are known): four lanes read a row's 64 bytes,
// so that a workgroup takes 64 rows at a time (32 rows of 128 bytes: a fifth more time), three or four rows each in
// flight; lanes and wavefronts add theirs in a fixed order.  A vector at the end moves down to end with
// the row, its first columns are another lane's.
struct ColumnSums {
    float *dweight, *dbias;
    int accumulate, blocks;
};
constexpr int kColumnLanes = 4;
template <typename XT, typename YT, int THREADS, bool CENTER>
__device__ __forceinline__ void column_sums(const NormArgs &a, const ColumnSums &to, int block)
{
    constexpr int EPV = kVec<XT>, kInFlight = EPV == 8 ? 3 : 4, kGroups = THREADS / kColumnLanes, kWaves = THREADS / kWave, kCols = kColumnLanes * EPV;
    __shared__ float part[kWaves][2][kCols];
    auto first_of = [&](int lane) { return (block * kColumnLanes + lane) * EPV; };
    auto at_of = [&](int lane) { return max(min(first_of(lane), a.H - EPV), 0); };
    const int lane = threadIdx.x % kColumnLanes, group = threadIdx.x / kColumnLanes, at = at_of(lane);
    float dw[EPV], db[EPV];
#pragma unroll
    for (int k = 0; k < EPV; ++k) dw[k] = db[k] = 0.0f;
    // (rows shorter than a vector are read by elements; which, is asked once: loads on either side of a branch are waited for there)
    auto sum_rows = [&](auto whole) {
        for (int64_t t0 = group; t0 < a.T; t0 += kGroups * kInFlight) {
            float x[kInFlight][EPV], g[kInFlight][EPV], rstd[kInFlight], mean[kInFlight];
#pragma unroll
            for (int j = 0; j < kInFlight; ++j) {
                const int64_t t = min(t0 + j * kGroups, a.T - 1);
                const char *row = static_cast<const char *>(a.x) + t * a.ldx * XT::kBytes;
                const char *grow = static_cast<const char *>(a.dy) + t * a.ldy * YT::kBytes;
                rstd[j] = a.rstd[t];
                mean[j] = CENTER ? a.mean[t] : 0.0f;
                if constexpr (whole) {
                    load_vec<XT, EPV>(row + at * XT::kBytes, x[j]);
                    load_vec<YT, EPV>(grow + at * YT::kBytes, g[j]);
                } else {
#pragma unroll
                    for (int k = 0; k < EPV; ++k) {
                        x[j][k] = load_elem<XT>(row, min(k, a.H - 1));
                        g[j][k] = load_elem<YT>(grow, min(k, a.H - 1));
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < kInFlight; ++j)
#pragma unroll
                for (int k = 0; k < EPV; ++k) {
                    const float v = t0 + j * kGroups < a.T ? g[j][k] : 0.0f;
                    dw[k] = fmaf(v, (CENTER ? x[j][k] - mean[j] : x[j][k]) * rstd[j], dw[k]);
                    if constexpr (CENTER) db[k] += v;
                }
        }
    };
    if (a.H >= EPV) sum_rows(std::true_type{});
    else sum_rows(std::false_type{});
#pragma unroll
    for (int k = 0; k < EPV; ++k)
#pragma unroll
        for (int off = kColumnLanes; off < kWave; off <<= 1) {
            dw[k] += __shfl_xor(dw[k], off, kWave);
            if constexpr (CENTER) db[k] += __shfl_xor(db[k], off, kWave);
        }
    if (threadIdx.x % kWave < kColumnLanes)
#pragma unroll
        for (int k = 0; k < EPV; ++k) {
            part[threadIdx.x / kWave][0][lane * EPV + k] = dw[k];
            if constexpr (CENTER) part[threadIdx.x / kWave][1][lane * EPV + k] = db[k];
        }
    __syncthreads();
    const int which = threadIdx.x / kCols, i = threadIdx.x % kCols, first = first_of(i / EPV), column = at_of(i / EPV) + i % EPV;
    float *out = which == 0 ? to.dweight : to.dbias;
    if (which > (CENTER ? 1 : 0) || !out || column < first || column >= a.H) return;
    float total = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += part[w][which][i];
    out[column] = to.accumulate ? out[column] + total : total;
}

// Each workgroup takes rows in turn and leaves its share of dw and db in partials [workgroup][dw | db][H]; a second
// kernel adds the shares in one order, so that identical inputs give identical sums.
// With to.blocks, that many workgroups come first that take the sums over rows, and no partial sums are left.
template <typename XT, typename YT, int LANES, int NV, bool CENTER>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void norm_bwd_kernel(NormArgs a, float *partials, ColumnSums to)
{
    if ((int)blockIdx.x < to.blocks) return column_sums<XT, YT, (LANES > 256 ? LANES : 256), CENTER>(a, to, (int)blockIdx.x);
    constexpr int EPV = kVec<XT>, kRows = LANES >= 256 ? 1 : 256 / LANES;
    // Five values for each of 32 elements a lane are 160 of its 256 registers, and 64-bit offsets of every vector in x and dy, which the
    // compiler computes ahead of the loop, were spilled (up to 29 registers, and loads then waited for one another): there they are
    // 32 bits from a base that is the workgroup's.  Layer norm, fp32 to bf16 4,096 x 16,384 184 -> 139 us, fp32 168 -> 161, bf16 to
    // fp32 4,096 x 16,000 149 -> 135; forms that have the registers are up to 6 % slower so (bf16 4,096 x 12,500 93 and 97).
    constexpr bool kTight = CENTER && LANES == 512 && NV * EPV == 32 && XT::kBytes + YT::kBytes > 4;
    __shared__ float red[2][2 * (LANES / kWave)];
    int phase = 0;
    const int lane = threadIdx.x % LANES, full = a.H / EPV, rest = a.H - full * EPV, group = kTight ? 0 : threadIdx.x / LANES;
    const int e_last = full * EPV + lane;
    const float inv_h = 1.0f / (float)a.H;
    const bool last = lane < rest;
    float w[NV][EPV], dw[NV][EPV], db[NV][EPV], w_last = 0.0f, dw_last = 0.0f, db_last = 0.0f;
    if (full)
#pragma unroll
        for (int i = 0; i < NV; ++i)
            load_param<EPV>(a.weight, a.param_f32, (int64_t)min(i * LANES + lane, full - 1) * EPV, 1.0f, w[i]);
    if (last) w_last = load_param(a.weight, a.param_f32, e_last, 1.0f);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int k = 0; k < EPV; ++k) dw[i][k] = db[i][k] = 0.0f;
    const int64_t stride = (int64_t)(gridDim.x - to.blocks) * kRows;
    for (int64_t t = (int64_t)(blockIdx.x - to.blocks) * kRows + group; t < a.T; t += stride) {
        const char *row = static_cast<const char *>(a.x) + t * a.ldx * XT::kBytes;
        const char *grow = static_cast<const char *>(a.dy) + t * a.ldy * YT::kBytes;
        char *out = static_cast<char *>(a.dx) + t * a.lddx * XT::kBytes;
        const float rstd = a.rstd[t], mean = CENTER ? a.mean[t] : 0.0f;
        float x[NV][EPV], g[NV][EPV], x_last = 0.0f, g_last = 0.0f;
        if (full)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int v = min(i * LANES + lane, full - 1);
                if constexpr (kTight) {
                    uint32_t here = (uint32_t)v;
                    asm volatile("" : "+v"(here));  // (not ahead of the loop)
                    load_vec<XT, EPV, true>(row + here * (uint32_t)(EPV * XT::kBytes), x[i]);
                    load_vec<YT, EPV, true>(grow + here * (uint32_t)(EPV * YT::kBytes), g[i]);
                } else {
                    load_vec<XT, EPV, true>(row + v * EPV * XT::kBytes, x[i]);
                    load_vec<YT, EPV, true>(grow + v * EPV * YT::kBytes, g[i]);
                }
            }
        if (last) {
            x_last = load_elem<XT>(row, e_last);
            g_last = load_elem<YT>(grow, e_last);
        }
        float s[2] = {0.0f, 0.0f};  // sums of g xhat and of g
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool on = i * LANES + lane < full;
#pragma unroll
            for (int k = 0; k < EPV; ++k) {
                x[i][k] = on ? (CENTER ? x[i][k] - mean : x[i][k]) * rstd : 0.0f;
                g[i][k] = on ? g[i][k] : 0.0f;
                dw[i][k] = fmaf(g[i][k], x[i][k], dw[i][k]);
                if constexpr (CENTER) db[i][k] += g[i][k];
                g[i][k] = on ? g[i][k] * w[i][k] : 0.0f;
                s[0] = fmaf(g[i][k], x[i][k], s[0]);
                if constexpr (CENTER) s[1] += g[i][k];
            }
        }
        if (last) {
            x_last = (x_last - mean) * rstd;
            dw_last = fmaf(g_last, x_last, dw_last);
            if constexpr (CENTER) db_last += g_last;
            g_last *= w_last;
            s[0] = fmaf(g_last, x_last, s[0]);
            if constexpr (CENTER) s[1] += g_last;
        }
        row_sum<LANES, 2>(s, red, phase);
        const float along = s[0] * inv_h, level = CENTER ? s[1] * inv_h : 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * LANES + lane;
            if (v < full) {
#pragma unroll
                for (int k = 0; k < EPV; ++k) g[i][k] = rstd * (g[i][k] - level - x[i][k] * along);
                store_vec<XT, EPV, true>(out + v * EPV * XT::kBytes, g[i]);
            }
        }
        if (last) store_elem<XT>(out, e_last, rstd * (g_last - level - x_last * along));
    }
    if (!partials) return;
    // the groups of lanes of this workgroup add their sums, one group after the other
    extern __shared__ __align__(16) float sums[];  // [dw | db][H rounded up to vectors], kRows > 1 only
    float *mine = partials + (int64_t)blockIdx.x * a.partial_rows * a.H;
    const int half = (a.H + 3) / 4 * 4;
    for (int r = 0; r < kRows; ++r) {
        if (r > 0) __syncthreads();
        if (group != r) continue;
        const bool first = r == 0, leave = r == kRows - 1;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * LANES + lane, e = v * EPV;
            if (v >= full) continue;
#pragma unroll
            for (int k = 0; k < EPV; k += 4) {
                typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
                f32x4_any p = {dw[i][k], dw[i][k + 1], dw[i][k + 2], dw[i][k + 3]};
                f32x4_any q = {db[i][k], db[i][k + 1], db[i][k + 2], db[i][k + 3]};
                if (!first) {
                    p += *reinterpret_cast<const f32x4_any *>(sums + e + k);
                    if constexpr (CENTER) q += *reinterpret_cast<const f32x4_any *>(sums + half + e + k);
                }
                if (leave) {
                    *reinterpret_cast<f32x4_any *>(mine + e + k) = p;
                    if (CENTER && a.partial_rows > 1) *reinterpret_cast<f32x4_any *>(mine + a.H + e + k) = q;
                } else {
                    *reinterpret_cast<f32x4_any *>(sums + e + k) = p;
                    if constexpr (CENTER) *reinterpret_cast<f32x4_any *>(sums + half + e + k) = q;
                }
            }
        }
        if (last) {
            const float p = dw_last + (first ? 0.0f : sums[e_last]), q = db_last + (first ? 0.0f : sums[half + e_last]);
            (leave ? mine : sums)[e_last] = p;
            if (!leave) sums[half + e_last] = q;
            else if (a.partial_rows > 1) mine[a.H + e_last] = q;
        }
    }
}

// columns of the partials, summed in order: a workgroup takes 32 columns, 32 runs of workgroups' shares each
__global__ __launch_bounds__(1024) void norm_bwd_sum_kernel(const float *partials, int parts, int64_t width, int64_t H,
                                                            float *dweight, float *dbias, int accumulate)
{
    __shared__ float part[32][33];
    const int col = threadIdx.x & 31, run = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + col;
    const int per = (parts + 31) / 32;
    float s = 0.0f;
    if (c < width) {
        const int end = min(parts, (run + 1) * per);
#pragma unroll 8
        for (int p = run * per; p < end; ++p) s += partials[(int64_t)p * width + c];
    }
    part[run][col] = s;
    __syncthreads();
    if (run == 0 && c < width) {
        float total = 0.0f;
#pragma unroll
        for (int r = 0; r < 32; ++r) total += part[r][col];
        float *to = c < H ? dweight : dbias;
        if (to) {
            to += c < H ? c : c - H;
            *to = accumulate ? *to + total : total;
        }
    }
}

template <typename XT, typename YT, int LANES, int NV>
hipError_t launch(const NormArgs &a, bool backward, float *partials, int64_t blocks, const ColumnSums &to, hipStream_t s)
{
    constexpr int kThreads = LANES > 256 ? LANES : 256;
    const dim3 grid((unsigned)(blocks + to.blocks)), block(kThreads);
    if (backward) {
        const size_t lds = LANES < 256 && partials ? (size_t)8 * ((a.H + 3) / 4 * 4) : 0;
        if (a.center) norm_bwd_kernel<XT, YT, LANES, NV, true><<<grid, block, lds, s>>>(a, partials, to);
        else norm_bwd_kernel<XT, YT, LANES, NV, false><<<grid, block, lds, s>>>(a, partials, to);
    } else if constexpr (XT::kBytes == 4 || LANES > 64 || NV < 4) {  // (the plan gives the forward pass no four of bf16)
        if (a.center) norm_fwd_kernel<XT, YT, LANES, NV, true><<<grid, block, 0, s>>>(a);
        else norm_fwd_kernel<XT, YT, LANES, NV, false><<<grid, block, 0, s>>>(a);
    }
    return hipGetLastError();
}

template <typename XT, typename YT>
hipError_t launch_of(const NormArgs &a, bool backward, float *partials, int64_t blocks, const ColumnSums &to, hipStream_t s)
{
    const NormPlan p = norm_plan(a.T, a.H, XT::kBytes, backward);
    // (norm_plan gives no other pair)
#define A3PO_NORM_CASE(L, N) \
    if (p.lanes == L && p.vectors == N) return launch<XT, YT, L, N>(a, backward, partials, blocks, to, s)
    A3PO_NORM_CASE(64, 1);
    A3PO_NORM_CASE(64, 2);
    A3PO_NORM_CASE(64, 3);
    A3PO_NORM_CASE(64, 4);
    if constexpr (XT::kBytes == 4) A3PO_NORM_CASE(64, 6);
    A3PO_NORM_CASE(256, 1);
    A3PO_NORM_CASE(256, 2);
    A3PO_NORM_CASE(256, 3);
    A3PO_NORM_CASE(256, 4);
    if constexpr (XT::kBytes == 2) A3PO_NORM_CASE(512, 3);
    A3PO_NORM_CASE(512, 4);
    if constexpr (XT::kBytes == 4) A3PO_NORM_CASE(512, 6);
    if constexpr (XT::kBytes == 4) A3PO_NORM_CASE(512, 8);
#undef A3PO_NORM_CASE
    return hipErrorInvalidValue;
}

hipError_t launch_any(const NormArgs &a, bool backward, float *partials, int64_t blocks, const ColumnSums &to, hipStream_t s)
{
    if (a.x_dt == A3PO_F32)
        return a.y_dt == A3PO_F32 ? launch_of<F32, F32>(a, backward, partials, blocks, to, s)
                                  : launch_of<F32, Bf16>(a, backward, partials, blocks, to, s);
    return a.y_dt == A3PO_F32 ? launch_of<Bf16, F32>(a, backward, partials, blocks, to, s)
                              : launch_of<Bf16, Bf16>(a, backward, partials, blocks, to, s);
}

}  // namespace

hipError_t launch_norm_fwd(const NormArgs &a, hipStream_t s)
{
    const NormPlan p = norm_plan(a.T, a.H, a.x_dt == A3PO_F32 ? 4 : 2, false);
    const int rows = p.lanes >= 256 ? 1 : 256 / p.lanes;
    const int64_t want = (a.T + rows - 1) / rows, most = 4096;
    return launch_any(a, false, nullptr, want < most ? want : most, ColumnSums{}, s);
}

hipError_t launch_norm_bwd(const NormArgs &a, float *dweight, float *dbias, int accumulate, void *workspace, hipStream_t s)
{
    const int x_bytes = a.x_dt == A3PO_F32 ? 4 : 2;
    const int64_t blocks = norm_bwd_blocks(a.T, a.H, x_bytes);
    NormArgs b = a;
    b.partial_rows = dbias ? 2 : 1;
    const bool sums = dweight || dbias;
    if (sums && norm_bwd_in_one(a.T, a.H, a.x, a.dy, a.dx)) {
        const int columns = kColumnLanes * 16 / x_bytes;
        return launch_any(b, true, nullptr, blocks, ColumnSums{dweight, dbias, accumulate, (a.H + columns - 1) / columns}, s);
    }
    float *partials = sums ? static_cast<float *>(workspace) : nullptr;
    if (a.T > 0)
        if (const hipError_t e = launch_any(b, true, partials, blocks, ColumnSums{}, s)) return e;
    if (!sums) return hipSuccess;
    const int64_t width = b.partial_rows * a.H;
    norm_bwd_sum_kernel<<<dim3((unsigned)((width + 31) / 32)), dim3(1024), 0, s>>>(
        partials, a.T > 0 ? (int)blocks : 0, width, a.H, dweight, dbias, accumulate);
    return hipGetLastError();
}

}  // namespace a3po
