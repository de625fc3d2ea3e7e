// Layer norm of rows, and its gradients.
//
//   m = mean(x),  r = 1 / sqrt(mean((x - m)^2) + eps),  y = (x - m) r w + b
//   h = (x - m) r,  u = w g:   dx = r (u - mean(u) - h mean(u h)),   dw = sum over rows of g h,   db = sum over rows of g
//
// Both directions are bound by memory: a row is read once, kept in the registers of a team of lanes, and written once.  Mean and
// squares are taken of (x - m) with the row at hand, so rows far from zero lose nothing; the few that fp32 cannot do are done again in fp64.  A team is as few lanes as hold the row
// in 16 to 32 elements each: few steps of a sum across lanes, and 64 bytes a lane in flight; more lanes where there are too few rows to fill the
// chip.  Teams keep the columns' parameters from row to row (a workgroup for every few rows instead: 52 -> 102 us for 507,001 x 100 in bf16).  Rows too
// long for 1,024 lanes are read again for each sum (2,048 x 40,000 in fp32 271, a copy 141).  us measured, and what the same bytes take a large copy: 507,001 x 100 in bf16 45 (44); gradients of
// 232,965 x 602 in fp32 347 (362), of 16,384 x 4,096 in bf16 82 (87).
//
// Gradients of weights: a team walks over every so-many-th row with the columns' sums in registers, a workgroup adds its teams' sums up in
// LDS and leaves one row of them, and a second launch adds these rows in a fixed order: the same inputs give the same bits.
#include <algorithm>
#include <exception>

#include "gp_internal.h"
#include "gp_rows.h"

namespace gp {

namespace {

struct NormArgs {
    const void* x;
    int64_t ldx, N;
    int d, nvec;
    const void *weight, *bias;
    int wide_weights;  // weights, bias and their gradients are fp32 (else bf16)
    float eps;
    double share;  // 1 / d
    void* y;
    int64_t ldy;
    float* stats;
};

struct NormGradArgs {
    const void *g, *x;
    int64_t ldg, ldx, N;
    int d, nvec;
    const float* stats;
    const void* weight;
    int wide_weights;
    void* x_grad;
    int64_t ldxg;
    void *weight_grad, *bias_grad;
    int accumulate;
    float* partial;  // [workgroups][2][d]: sums of g h, sums of g
    float* means;    // long rows: [N][2], mean(u) and mean(u h)
    int64_t chunk;   // long rows: rows that one workgroup sums up
    unsigned row_blocks;  // workgroups that have rows; those behind them have columns
};

__device__ __forceinline__ float parameter(const void* p, int wide, int i, float without)
{
    return !p ? without : wide ? ((const float*)p)[i] : widen(((const bf16_t*)p)[i]);
}

// VEC of them from place i on (16 bytes a request, whatever the place)
template <int VEC>
__device__ __forceinline__ void parameters(const void* p, int wide, int i, float without, float (&v)[VEC])
{
    if (!p) {
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[k] = without;
    } else if (wide) {
        load_vec<float, VEC>((const float*)p + i, v);
    } else {
        load_vec<bf16_t, VEC>((const bf16_t*)p + i, v);
    }
}

// The sum over a team of TPR lanes: of a part of a wavefront, or of a whole workgroup, whose `lds` (a float per wavefront) nothing else touches until
// every wavefront has passed a later barrier.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* lds)
{
    if constexpr (TPR <= 64) {
        return team_sum<TPR>(v);
    } else {
        v = team_sum<64>(v);
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        return team_sum<TPR / 64>(lds[threadIdx.x & (TPR / 64 - 1)]);
    }
}

// ---- forward ----------------------------------------------------------------------------------------------------

// Lanes of a workgroup: teams of a wavefront or less come several to one, longer ones alone, since they meet at barriers.
template <int TPR>
constexpr int kNormBlock = TPR <= 64 ? 256 : TPR;

// Wavefronts of a SIMD that a kernel is built for, by the types and the elements of a row that a lane holds: a launch is of eight workgroups of four to a compute
// unit, and takes longer where they come in other rounds (us, five at a time / four: 492,307 x 130 in bf16 68 / 62, 15,609 x 4100 61.6 / 55.3).
template <typename TX, typename TY, int E>
constexpr int kNormWaves = E <= 12 ? 8 : E <= 16 ? (sizeof(TX) == sizeof(TY) ? 6 : 5) : E <= 24 || sizeof(TY) == 2 ? 4 : 3;

// Whether a row's variance (with eps) is not to be had from sums in fp32: squares or sums beyond it (from |x - m| of 2^64 / sqrt(d) on, or an infinity or NaN),
// or nothing but the rounding of its first mean, `rest` off, whose square is taken off it and known to 2^-17 or so: rows of one value far from zero.
__device__ __forceinline__ bool beyond_fp32(float v, float rest) { return !(v < __builtin_inff()) || rest * rest > 32.0f * v; }

// Such a row: its sums in fp64, element by element from memory, a lane writing what it has read.  A row of one value is told by its variance, which is 0 or
// 2^-63 of the mean's square and more where elements are 24 bits: below 2^-80 of it is what the mean's rounding left.  An infinity or NaN makes all NaN.  It
// is rare, and takes as few registers as it can beside what the others keep: loops as they stand, no division or root in fp64.
template <int TPR>
__device__ __forceinline__ double far_sum(double v, int thread, double* lds)
{
#pragma unroll 1
    for (int m = 4; m < (TPR < 64 ? TPR : 64) * 4; m *= 2) {
        const uint64_t bits = __builtin_bit_cast(uint64_t, v);
        const unsigned low = __builtin_amdgcn_ds_bpermute((thread << 2) ^ m, (int)bits), high = __builtin_amdgcn_ds_bpermute((thread << 2) ^ m, (int)(bits >> 32));
        v += __builtin_bit_cast(double, (uint64_t)high << 32 | low);
    }
    if constexpr (TPR > 64) {
        __syncthreads();  // (whoever still reads the last sum)
        if ((thread & 63) == 0) lds[thread >> 6] = v;
        __syncthreads();
        v = 0.0;
#pragma unroll 1
        for (int i = 0; i < TPR / 64; ++i) v += lds[i];
    }
    return v;
}
template <typename TX, typename TY, int TPR>
__device__ __forceinline__ void norm_far_row(const NormArgs& a, int64_t row, double* lds)
{
    int thread = threadIdx.x;
    asm volatile("" : "+v"(thread));  // (so that nothing of it is worked out ahead and kept from row to row)
    const int lane = thread % TPR;
    const TX* const x = (const TX*)a.x + row * a.ldx;
    TY* const y = (TY*)a.y + row * a.ldy;
    double sum = 0.0, rest = 0.0, squares = 0.0;
#pragma unroll 1
    for (int64_t j = lane; j < a.d; j += TPR) sum += widen(x[j]);
    const double mean = far_sum<TPR>(sum, thread, lds) * a.share;
#pragma unroll 1
    for (int64_t j = lane; j < a.d; j += TPR) {
        const double e = widen(x[j]) - mean;
        rest += e, squares += e * e;
    }
    rest = far_sum<TPR>(rest, thread, lds) * a.share;
    double v = far_sum<TPR>(squares, thread, lds) * a.share - rest * rest;
    const bool flat = v <= mean * mean * 0x1p-80;
    v = (flat ? 0.0 : v) + a.eps;
    double r = __builtin_amdgcn_rsq(v);  // (to 24 bits or more, 47 by one step)
    r *= 1.5 - 0.5 * v * r * r;
#pragma unroll 1
    for (int64_t j = lane; j < a.d; j += TPR) {
        const float h = flat ? 0.0f : (float)(((widen(x[j]) - mean) - rest) * r);
        y[j] = narrow<TY>(h * parameter(a.weight, a.wide_weights, (int)j, 1.0f) + parameter(a.bias, a.wide_weights, (int)j, 0.0f));
    }
    if (a.stats && lane == 0) a.stats[2 * row] = (float)(mean + rest), a.stats[2 * row + 1] = (float)r;
}

// Vector t = v * TPR + lane of a row starts at column t * VEC; the last one is moved back to end with the row, and its first elements, which the
// vector before has as well, take no part in sums.  NV is as small as holds the row, so only vectors v = NV - 1 may be that one or none.
// y may be x: a row is read before it is written.
template <typename TX, typename TY, int VEC, int NV, int TPR>
__global__ __launch_bounds__(kNormBlock<TPR>) __attribute__((amdgpu_waves_per_eu(kNormWaves<TX, TY, NV * VEC>, kNormWaves<TX, TY, NV * VEC>))) void gp_norm_rows(NormArgs a)
{
    constexpr int TEAMS = kNormBlock<TPR> / TPR;
    __shared__ float lds[3][16];
    __shared__ double wide[TPR > 64 ? TPR / 64 : 1];
    const int lane = threadIdx.x % TPR;
    float w[NV][VEC], b[NV][VEC];
    int col[NV], first = 0;  // the first element of vector NV - 1 that counts
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int t = v * TPR + lane;
        col[v] = t < a.nvec ? min(t * VEC, a.d - VEC) : 0;
        if (v == NV - 1) first = t < a.nvec ? t * VEC - col[v] : VEC;
        parameters<VEC>(a.weight, a.wide_weights, col[v], 1.0f, w[v]);
        parameters<VEC>(a.bias, a.wide_weights, col[v], 0.0f, b[v]);
    }
    const float share = 1.0f / (float)a.d;
    for (int64_t row = (int64_t)blockIdx.x * TEAMS + threadIdx.x / TPR; row < a.N; row += (int64_t)gridDim.x * TEAMS) {
        const TX* const x = (const TX*)a.x + row * a.ldx;
        float e[NV][VEC], sum = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) load_vec<TX, VEC>(x + col[v], e[v]);
        // all of a row is asked for before any of it is used; where registers are tight the compiler's own order is better (us, with / without: 492,307 x 130 in
        // fp32 112.5 / 119.2, in bf16 61.4 / 65.2; 16,384 x 4,096 in bf16 56.3 / 54.4, 30,000 x 3000 80.6 / 76.8)
        if constexpr (sizeof(TX) == 4 || (NV <= 3 && TPR <= 64)) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum += v < NV - 1 || i >= first ? e[v][i] : 0.0f;
        const float about = row_sum<TPR>(sum, lds[0]) * share;
        float rest = 0.0f, squares = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                e[v][i] -= about;
                rest += v < NV - 1 || i >= first ? e[v][i] : 0.0f;
                squares += v < NV - 1 || i >= first ? e[v][i] * e[v][i] : 0.0f;
            }
        // the mean again, of what is left: a sum of values far from zero is off by many times what one of them is
        rest = row_sum<TPR>(rest, lds[1]) * share;
        const float variance = row_sum<TPR>(squares, lds[2]) * share - rest * rest, v = (variance < 0.0f ? 0.0f : variance) + a.eps;
        if (__builtin_expect(beyond_fp32(v, rest), 0)) {  // (all lanes of a team alike)
            norm_far_row<TX, TY, TPR>(a, row, wide);
            continue;
        }
        const float r = 1.0f / sqrtf(v);
        TY* const y = (TY*)a.y + row * a.ldy;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) e[v][i] = (e[v][i] - rest) * r * w[v][i] + b[v][i];
            if (v < NV - 1 || first < VEC) store_vec<TY, VEC>(y + col[v], e[v]);
        }
        if (a.stats && lane == 0) a.stats[2 * row] = about + rest, a.stats[2 * row + 1] = r;
    }
}

// The sum over a workgroup of 1,024, in fp64 (a lane of a long row adds up many terms).
__device__ __forceinline__ double workgroup_sum(double v, double* lds)
{
#pragma unroll
    for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m, 64);
    __syncthreads();  // (whoever still reads the last sum)
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += lds[i];
    return s;
}

// Rows too long for registers: a workgroup reads one three times.  The mean is taken off in two parts, rounded to fp32 and what that left: a row far from zero
// would lose half a step of its mean, times r, otherwise (us, in two parts / in one: 2,048 x 40,000 in fp32 271.2 / 270.9, in bf16 233.8 / 233.2).
template <typename TX, typename TY>
__global__ __launch_bounds__(1024) void gp_norm_long(NormArgs a)
{
    __shared__ double lds[16];
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const TX* const x = (const TX*)a.x + row * a.ldx;
        double sum = 0.0;
        for (int64_t j = threadIdx.x; j < a.d; j += 1024) sum += widen(x[j]);
        const double m = workgroup_sum(sum, lds) / a.d;
        const float mean = (float)m, rest = (float)(m - mean);
        double squares = 0.0;
        for (int64_t j = threadIdx.x; j < a.d; j += 1024) {
            const float e = (widen(x[j]) - mean) - rest;
            squares += e * e;
        }
        const float v = (float)(workgroup_sum(squares, lds) / a.d) + a.eps;
        if (beyond_fp32(v, rest)) {
            norm_far_row<TX, TY, 1024>(a, row, lds);
            continue;
        }
        const float r = 1.0f / sqrtf(v);
        TY* const y = (TY*)a.y + row * a.ldy;
        for (int64_t j = threadIdx.x; j < a.d; j += 1024)
            y[j] = narrow<TY>(((widen(x[j]) - mean) - rest) * r * parameter(a.weight, a.wide_weights, (int)j, 1.0f) + parameter(a.bias, a.wide_weights, (int)j, 0.0f));
        if (a.stats && threadIdx.x == 0) a.stats[2 * row] = mean, a.stats[2 * row + 1] = r;
    }
}

// ---- backward -----------------------------------------------------------------------------------------------------

__device__ __forceinline__ void write_sum(const NormGradArgs& a, bool of_weight, int64_t at, float sum)
{
    void* const to = of_weight ? a.weight_grad : a.bias_grad;
    if (!to) return;
    if (a.wide_weights)
        ((float*)to)[at] = sum + (a.accumulate ? ((float*)to)[at] : 0.0f);
    else
        ((bf16_t*)to)[at] = narrow<bf16_t>(sum + (a.accumulate ? widen(((bf16_t*)to)[at]) : 0.0f));
}

// The sums of eight columns down all rows, by a workgroup: few rows are read once more from the caches sooner than a second launch has begun.
template <typename TX, typename TG, int BLOCK>
__device__ __forceinline__ void sum_columns(const NormGradArgs& a, unsigned block)
{
    __shared__ float sums[2][BLOCK / 64][8];
    const int c = threadIdx.x & 7;
    const int64_t j = (int64_t)block * 8 + c, at = min(j, (int64_t)a.d - 1);
    float dw = 0.0f, db = 0.0f;
#pragma unroll 4
    for (int64_t row = threadIdx.x >> 3; row < a.N; row += BLOCK / 8) {
        const float mean = a.stats[2 * row], r = a.stats[2 * row + 1];
        const float g = widen(((const TG*)a.g)[row * a.ldg + at]), h = (widen(((const TX*)a.x)[row * a.ldx + at]) - mean) * r;
        dw += g * h, db += g;
    }
#pragma unroll
    for (int m = 8; m < 64; m *= 2) dw += __shfl_xor(dw, m, 64), db += __shfl_xor(db, m, 64);
    if ((threadIdx.x & 63) < 8) sums[0][threadIdx.x >> 6][c] = dw, sums[1][threadIdx.x >> 6][c] = db;
    __syncthreads();
    if (threadIdx.x >= 16 || j >= a.d) return;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < BLOCK / 64; ++w) sum += sums[threadIdx.x >> 3][w][c];
    write_sum(a, threadIdx.x < 8, j, sum);
}

// x_grad may be x or g: a row is read before it is written.
template <typename TX, typename TG, int VEC, int NV, int TPR>
__global__ __launch_bounds__(TPR < 512 ? 512 : TPR) void gp_norm_grad_rows(NormGradArgs a)
{
    constexpr int BLOCK = TPR < 512 ? 512 : TPR, TEAMS = BLOCK / TPR;
    constexpr int WAVE = TPR < 64 ? TPR : 64;  // lanes of a wavefront that hold different columns
    constexpr int SETS = TPR < 64 ? BLOCK / 64 : TEAMS;  // sets of columns' sums that are left after a wavefront has added up its own
    __shared__ float lds[2][2][16];
    extern __shared__ float sums[];  // [SETS][2][NV * VEC][TPR] where SETS > 1
    if (blockIdx.x >= a.row_blocks) {
        sum_columns<TX, TG, BLOCK>(a, blockIdx.x - a.row_blocks);
        return;
    }
    const int lane = threadIdx.x % TPR;
    float w[NV][VEC], dw[NV][VEC] = {}, db[NV][VEC] = {};
    int col[NV], first = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int t = v * TPR + lane;
        col[v] = t < a.nvec ? min(t * VEC, a.d - VEC) : 0;
        if (v == NV - 1) first = t < a.nvec ? t * VEC - col[v] : VEC;
        parameters<VEC>(a.weight, a.wide_weights, col[v], 1.0f, w[v]);
    }
    const float share = 1.0f / (float)a.d;
    int turn = 0;
    // (every team of a workgroup goes round as often: long ones meet at a barrier)
    for (int64_t base = (int64_t)blockIdx.x * TEAMS; base < a.N; base += (int64_t)a.row_blocks * TEAMS, turn ^= 1) {
        const int64_t row = base + threadIdx.x / TPR;
        const bool live = row < a.N;
        float h[NV][VEC], u[NV][VEC], su = 0.0f, suh = 0.0f, r = 0.0f;
        if (live) {
            const TX* const x = (const TX*)a.x + row * a.ldx;
            const TG* const g = (const TG*)a.g + row * a.ldg;
            const float mean = a.stats[2 * row];
            r = a.stats[2 * row + 1];
#pragma unroll
            for (int v = 0; v < NV; ++v) load_vec<TX, VEC>(x + col[v], h[v]), load_vec<TG, VEC>(g + col[v], u[v]);
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    h[v][i] = (h[v][i] - mean) * r;
                    db[v][i] += u[v][i];
                    dw[v][i] += u[v][i] * h[v][i];
                    u[v][i] *= w[v][i];
                    su += v < NV - 1 || i >= first ? u[v][i] : 0.0f;
                    suh += v < NV - 1 || i >= first ? u[v][i] * h[v][i] : 0.0f;
                }
        }
        if constexpr (TPR <= 64) {
            su = team_sum<TPR>(su) * share, suh = team_sum<TPR>(suh) * share;
        } else {
            su = team_sum<64>(su), suh = team_sum<64>(suh);
            if ((threadIdx.x & 63) == 0) lds[turn][0][threadIdx.x >> 6] = su, lds[turn][1][threadIdx.x >> 6] = suh;
            __syncthreads();
            const int at = threadIdx.x / TPR * (TPR / 64) + (threadIdx.x & (TPR / 64 - 1));
            su = team_sum<TPR / 64>(lds[turn][0][at]) * share, suh = team_sum<TPR / 64>(lds[turn][1][at]) * share;
        }
        if (!live || !a.x_grad) continue;
        TX* const out = (TX*)a.x_grad + row * a.ldxg;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) u[v][i] = r * (u[v][i] - su - h[v][i] * suh);
            if (v < NV - 1 || first < VEC) store_vec<TX, VEC>(out + col[v], u[v]);
        }
    }
    if (!a.partial) return;
    // the teams of a wavefront, by halves; then the sets, in order
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < VEC; ++i)
#pragma unroll
            for (int m = WAVE; m < 64; m *= 2) dw[v][i] += __shfl_xor(dw[v][i], m, 64), db[v][i] += __shfl_xor(db[v][i], m, 64);
    float* const out = a.partial + (int64_t)blockIdx.x * 2 * a.d;
    if constexpr (SETS > 1) {
        if (TPR >= 64 || (threadIdx.x & 63) < TPR) {
            float* const mine = sums + (threadIdx.x / (TPR < 64 ? 64 : TPR)) * (2 * NV * VEC * TPR) + lane;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < VEC; ++i) mine[(v * VEC + i) * TPR] = dw[v][i], mine[(NV * VEC + v * VEC + i) * TPR] = db[v][i];
        }
        __syncthreads();
        for (int j = threadIdx.x; j < 2 * a.d; j += BLOCK) {
            const int c = j < a.d ? j : j - a.d, t = min(c / VEC, a.nvec - 1), start = min(t * VEC, a.d - VEC);
            const int place = ((j < a.d ? 0 : NV * VEC) + t / TPR * VEC + (c - start)) * TPR + t % TPR;
            float s = 0.0f;
#pragma unroll
            for (int k = 0; k < SETS; ++k) s += sums[k * (2 * NV * VEC * TPR) + place];
            out[j] = s;
        }
    } else {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (v < NV - 1 || i >= first) out[col[v] + i] = dw[v][i], out[a.d + col[v] + i] = db[v][i];
    }
}

// Adds up the workgroups' sums: 32 columns by 32 stretches of rows to a workgroup, each stretch in order, the stretches by halves.
__global__ __launch_bounds__(1024) void gp_norm_grad_join(NormGradArgs a, int64_t rows)
{
    __shared__ float lds[32][33];
    const int c = threadIdx.x & 31, s = threadIdx.x >> 5;
    const int64_t width = 2 * (int64_t)a.d;
    for (int64_t first = (int64_t)blockIdx.x * 32; first < width; first += (int64_t)gridDim.x * 32) {
        const int64_t j = first + c;
        float sum = 0.0f;
        if (j < width) {
            int64_t k = s;
            for (; k + 96 < rows; k += 128) {
                const float p = a.partial[k * width + j], q = a.partial[(k + 32) * width + j], t = a.partial[(k + 64) * width + j], o = a.partial[(k + 96) * width + j];
                sum += (p + q) + (t + o);
            }
            for (; k < rows; k += 32) sum += a.partial[k * width + j];
        }
        lds[s][c] = sum;
        __syncthreads();
        if (s == 0 && j < width) {
            float part[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) part[i] = lds[i][c];
#pragma unroll
            for (int n = 16; n > 0; n /= 2)
#pragma unroll
                for (int i = 0; i < n; ++i) part[i] += part[i + n];
            write_sum(a, j < a.d, j < a.d ? j : j - a.d, part[0]);
        }
        __syncthreads();
    }
}

// Rows too long for registers, first half: mean(u) and mean(u h) of a row.
template <typename TX, typename TG>
__global__ __launch_bounds__(1024) void gp_norm_grad_means(NormGradArgs a)
{
    __shared__ double lds[16];
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const TX* const x = (const TX*)a.x + row * a.ldx;
        const TG* const g = (const TG*)a.g + row * a.ldg;
        const float mean = a.stats[2 * row], r = a.stats[2 * row + 1];
        double su = 0.0, suh = 0.0;
        for (int64_t j = threadIdx.x; j < a.d; j += 1024) {
            const float u = widen(g[j]) * parameter(a.weight, a.wide_weights, (int)j, 1.0f);
            su += u, suh += u * ((widen(x[j]) - mean) * r);
        }
        su = workgroup_sum(su, lds), suh = workgroup_sum(suh, lds);
        if (threadIdx.x == 0) a.means[2 * row] = (float)(su / a.d), a.means[2 * row + 1] = (float)(suh / a.d);
    }
}

// Second half: a column per lane, down a stretch of rows.
template <typename TX, typename TG>
__global__ __launch_bounds__(256) void gp_norm_grad_columns(NormGradArgs a)
{
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= a.d) return;
    const float w = parameter(a.weight, a.wide_weights, (int)j, 1.0f);
    float dw = 0.0f, db = 0.0f;
    const int64_t from = blockIdx.y * a.chunk, to = min(from + a.chunk, a.N);
    for (int64_t row = from; row < to; ++row) {
        const float mean = a.stats[2 * row], r = a.stats[2 * row + 1];
        const float g = widen(((const TG*)a.g)[row * a.ldg + j]), h = (widen(((const TX*)a.x)[row * a.ldx + j]) - mean) * r;
        dw += g * h, db += g;
        if (a.x_grad) ((TX*)a.x_grad)[row * a.ldxg + j] = narrow<TX>(r * (g * w - a.means[2 * row] - h * a.means[2 * row + 1]));
    }
    if (!a.partial) return;
    a.partial[blockIdx.y * 2 * (int64_t)a.d + j] = dw;
    a.partial[blockIdx.y * 2 * (int64_t)a.d + a.d + j] = db;
}

// ---- host ----------------------------------------------------------------------------------------------------------

constexpr int64_t kMaxBlocks = 1 << 20;  // of a launch; workgroups walk on through the rest
constexpr int64_t kUnits = 256;          // compute units
constexpr int64_t kFull = kUnits * 16;   // wavefronts below which a row is spread over more lanes
constexpr int kMostLanes = 1024;
constexpr int kGradElements = 16;        // of a row and lane in the backward pass, which holds it, its gradient, the weights and two sums of each
constexpr int kLongRow = kMostLanes * kGradElements;
constexpr int64_t kLongChunks = 64;      // stretches of rows that long rows' weight gradients are summed in

// Lanes of a row's team: as few as hold it in `most` vectors each; more, up to a wavefront, where the rows make too few wavefronts.
int team_lanes(int64_t N, int64_t nvec, int most)
{
    int lanes = 2;
    while (lanes < kMostLanes && nvec > (int64_t)lanes * most) lanes *= 2;
    while (lanes < 64 && nvec > lanes && N * lanes / 64 < kFull) lanes *= 2;
    return lanes;
}

template <typename TX, typename TY, int VEC, int NV, int TPR>
gp_status launch_norm(const NormArgs& a, hipStream_t stream)
{
    constexpr int BLOCK = kNormBlock<TPR>, TEAMS = BLOCK / TPR;
    const int64_t blocks = std::min((a.N + TEAMS - 1) / TEAMS, kUnits * 2048 / BLOCK);
    profile_begin("gp_norm_rows", stream);
    hipLaunchKernelGGL((gp_norm_rows<TX, TY, VEC, NV, TPR>), dim3((unsigned)blocks), dim3(BLOCK), 0, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    return GP_OK;
}
template <typename TX, typename TY, int VEC, int TPR>
gp_status launch_norm(const NormArgs& a, hipStream_t stream)
{
    switch ((a.nvec + TPR - 1) / TPR) {
    case 1: return launch_norm<TX, TY, VEC, 1, TPR>(a, stream);
    case 2: return launch_norm<TX, TY, VEC, 2, TPR>(a, stream);
    case 3: return launch_norm<TX, TY, VEC, 3, TPR>(a, stream);
    default: return launch_norm<TX, TY, VEC, 4, TPR>(a, stream);
    }
}
template <typename TX, typename TY>
gp_status launch_norm(NormArgs a, hipStream_t stream)
{
    constexpr int VEC = 16 / sizeof(TX);
    if (a.d < VEC) {
        a.nvec = a.d;
        return launch_norm<TX, TY, 1, 1, 8>(a, stream);
    }
    if (a.d > kMostLanes * 4 * VEC) {
        profile_begin("gp_norm_long", stream);
        hipLaunchKernelGGL((gp_norm_long<TX, TY>), dim3((unsigned)std::min(a.N, kMaxBlocks)), dim3(1024), 0, stream, a);
        profile_end(stream);
        GP_HIP(hipGetLastError());
        return GP_OK;
    }
    a.nvec = (a.d + VEC - 1) / VEC;
    // four vectors to a lane; two of narrow rows in bf16, whose parameters take more registers than the row (us, two / four: 507,001 x 100 48 / 54,
    // 492,307 x 130 64 / 62, 64,000 x 1000 54 / 51, 62,135 x 1030 82 / 54, 15,609 x 4100 80 / 56)
    switch (team_lanes(a.N, a.nvec, sizeof(TX) == 2 && a.nvec <= 16 ? 2 : 4)) {
    case 2: return launch_norm<TX, TY, VEC, 2>(a, stream);
    case 4: return launch_norm<TX, TY, VEC, 4>(a, stream);
    case 8: return launch_norm<TX, TY, VEC, 8>(a, stream);
    case 16: return launch_norm<TX, TY, VEC, 16>(a, stream);
    case 32: return launch_norm<TX, TY, VEC, 32>(a, stream);
    case 64: return launch_norm<TX, TY, VEC, 64>(a, stream);
    case 128: return launch_norm<TX, TY, VEC, 128>(a, stream);
    case 256: return launch_norm<TX, TY, VEC, 256>(a, stream);
    case 512: return launch_norm<TX, TY, VEC, 512>(a, stream);
    default: return launch_norm<TX, TY, VEC, 1024>(a, stream);
    }
}

// Few rows: their columns are summed by workgroups of their own in the same launch.  us on the GPU, one launch / rows' sums and a second one: 64 x 128
// 3.5 / 5.8, 1000 x 256 4.9 / 6.9, 300 x 1000 5.3 / 8.6, 1000 x 1000 8.6 / 10.1, 128 x 8000 11.2 / 15.4; 2048 x 128 6.4 / 6.2, 2048 x 500 11.9 / 8.5 (fp32).
bool few_rows(int64_t N, int64_t d) { return N <= 1024 && N * d <= (1 << 20); }

// Workgroups of the backward pass, a row of sums each: two of 512 or one of 1,024 to a compute unit, fewer where rows are.
template <int TPR>
constexpr int kGradBlock = TPR < 512 ? 512 : TPR;
template <int TPR>
int64_t grad_blocks(int64_t N)
{
    constexpr int TEAMS = kGradBlock<TPR> / TPR;
    // (and eight rows to a team, or one workgroup to a unit: rows of sums are written and read again; 2000 x 5000 in bf16 32 -> 28 us, 3000 x 1000 14 -> 11.5)
    return std::min({(N + TEAMS - 1) / TEAMS, kUnits * 1024 / kGradBlock<TPR>, std::max(kUnits, (N + TEAMS * 8 - 1) / (TEAMS * 8))});
}

gp_status launch_join(const NormGradArgs& a, int64_t rows, hipStream_t stream)
{
    if (!a.weight_grad && !a.bias_grad) return GP_OK;
    profile_begin("gp_norm_grad_join", stream);
    hipLaunchKernelGGL(gp_norm_grad_join, dim3((unsigned)std::min((2 * (int64_t)a.d + 31) / 32, kMaxBlocks)), dim3(1024), 0, stream, a, rows);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    return GP_OK;
}

template <typename TX, typename TG, int VEC, int NV, int TPR>
gp_status launch_grad_rows(const NormGradArgs& a, unsigned blocks, size_t lds, hipStream_t stream)
{
    profile_begin("gp_norm_grad_rows", stream);
    hipLaunchKernelGGL((gp_norm_grad_rows<TX, TG, VEC, NV, TPR>), dim3(blocks), dim3(kGradBlock<TPR>), lds, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    return GP_OK;
}
template <typename TX, typename TG, int VEC, int NV, int TPR>
gp_status launch_norm_grad(NormGradArgs a, hipStream_t stream)
{
    constexpr int BLOCK = kGradBlock<TPR>, TEAMS = BLOCK / TPR, SETS = TPR < 64 ? BLOCK / 64 : TEAMS;
    constexpr size_t lds = SETS > 1 ? (size_t)SETS * 2 * NV * VEC * TPR * 4 : 0;
    const unsigned blocks = (unsigned)grad_blocks<TPR>(a.N), columns = a.weight_grad || a.bias_grad ? (unsigned)((a.d + 7) / 8) : 0;
    if (few_rows(a.N, a.d)) {
        a.partial = nullptr;
        gp_status st = GP_OK;
        if (columns && (a.x_grad == a.x || a.x_grad == a.g)) {  // what the columns' workgroups read, rows' would write: one after the other
            a.row_blocks = 0;
            st = launch_grad_rows<TX, TG, VEC, NV, TPR>(a, columns, 0, stream);
            a.row_blocks = blocks;
            return st == GP_OK ? launch_grad_rows<TX, TG, VEC, NV, TPR>(a, blocks, 0, stream) : st;
        }
        a.row_blocks = a.x_grad ? blocks : 0;
        return launch_grad_rows<TX, TG, VEC, NV, TPR>(a, a.row_blocks + columns, 0, stream);
    }
    if constexpr (lds > 0) {
        gp_status st = raise_lds<&gp_norm_grad_rows<TX, TG, VEC, NV, TPR>>(lds);
        if (st != GP_OK) return st;
    }
    a.row_blocks = blocks;
    gp_status st = launch_grad_rows<TX, TG, VEC, NV, TPR>(a, blocks, lds, stream);
    return st == GP_OK ? launch_join(a, blocks, stream) : st;
}
template <typename TX, typename TG, int VEC, int TPR>
gp_status launch_norm_grad(const NormGradArgs& a, hipStream_t stream)
{
    const int need = (a.nvec + TPR - 1) / TPR;
    if (need == 1) return launch_norm_grad<TX, TG, VEC, 1, TPR>(a, stream);
    if constexpr (VEC * 4 <= kGradElements) {
        if (need == 3) return launch_norm_grad<TX, TG, VEC, 3, TPR>(a, stream);
        if (need == 4) return launch_norm_grad<TX, TG, VEC, 4, TPR>(a, stream);
    }
    return launch_norm_grad<TX, TG, VEC, 2, TPR>(a, stream);
}
template <typename TX, typename TG>
gp_status launch_norm_grad(NormGradArgs a, hipStream_t stream)
{
    constexpr int VEC = 16 / sizeof(TX);
    if (a.d < VEC) {
        a.nvec = a.d;
        return launch_norm_grad<TX, TG, 1, 1, 8>(a, stream);
    }
    if (a.d > kLongRow) {
        profile_begin("gp_norm_grad_means", stream);
        hipLaunchKernelGGL((gp_norm_grad_means<TX, TG>), dim3((unsigned)std::min(a.N, kMaxBlocks)), dim3(1024), 0, stream, a);
        profile_end(stream);
        GP_HIP(hipGetLastError());
        const int64_t chunks = std::min(a.N, kLongChunks);
        a.chunk = (a.N + chunks - 1) / chunks;
        const int64_t used = (a.N + a.chunk - 1) / a.chunk;
        profile_begin("gp_norm_grad_columns", stream);
        hipLaunchKernelGGL((gp_norm_grad_columns<TX, TG>), dim3((unsigned)(((int64_t)a.d + 255) / 256), (unsigned)used), dim3(256), 0, stream, a);
        profile_end(stream);
        GP_HIP(hipGetLastError());
        return launch_join(a, used, stream);
    }
    a.nvec = (a.d + VEC - 1) / VEC;
    switch (team_lanes(a.N, a.nvec, kGradElements / VEC)) {
    case 2: return launch_norm_grad<TX, TG, VEC, 2>(a, stream);
    case 4: return launch_norm_grad<TX, TG, VEC, 4>(a, stream);
    case 8: return launch_norm_grad<TX, TG, VEC, 8>(a, stream);
    case 16: return launch_norm_grad<TX, TG, VEC, 16>(a, stream);
    case 32: return launch_norm_grad<TX, TG, VEC, 32>(a, stream);
    case 64: return launch_norm_grad<TX, TG, VEC, 64>(a, stream);
    case 128: return launch_norm_grad<TX, TG, VEC, 128>(a, stream);
    case 256: return launch_norm_grad<TX, TG, VEC, 256>(a, stream);
    case 512: return launch_norm_grad<TX, TG, VEC, 512>(a, stream);
    default: return launch_norm_grad<TX, TG, VEC, 1024>(a, stream);
    }
}

bool known(gp_dtype t) { return t == GP_F32 || t == GP_BF16; }

gp_status layer_norm(const void* x, int64_t ldx, gp_dtype dtype, int64_t N, int32_t d, const void* weight, const void* bias, gp_dtype weight_dtype,
                     float eps, void* y, int64_t ldy, gp_dtype out_dtype, float* stats, hipStream_t stream)
{
    if (!known(dtype) || !known(weight_dtype) || !known(out_dtype))
        return fail(GP_ERR_INVALID_ARG, "unknown dtype %d, %d, %d", (int)dtype, (int)weight_dtype, (int)out_dtype);
    if (N < 0 || d < 1 || ldx < d || ldy < d) return fail(GP_ERR_INVALID_ARG, "need N >= 0, d >= 1, ldx >= d, ldy >= d");
    if (!(eps > 0.0f) || eps > 1e30f) return fail(GP_ERR_INVALID_ARG, "need a finite eps above 0");
    if (N == 0) return GP_OK;
    if (!x || !y) return fail(GP_ERR_INVALID_ARG, "NULL argument");
    NormArgs a{};
    a.x = x, a.ldx = ldx, a.N = N, a.d = d, a.weight = weight, a.bias = bias, a.wide_weights = weight_dtype == GP_F32, a.eps = eps, a.share = 1.0 / d, a.y = y, a.ldy = ldy,
    a.stats = stats;
    if (dtype == GP_F32) return out_dtype == GP_F32 ? launch_norm<float, float>(a, stream) : launch_norm<float, bf16_t>(a, stream);
    return out_dtype == GP_F32 ? launch_norm<bf16_t, float>(a, stream) : launch_norm<bf16_t, bf16_t>(a, stream);
}

struct NormGradLayout {
    int64_t partial, total;
};
// rows of sums: of the most workgroups that any team makes of N rows (teams of 8 lanes come 64 to a workgroup, those of 512 or more one)
NormGradLayout norm_grad_layout(int64_t N, int32_t d)
{
    const int64_t rows = d > kLongRow ? std::min(N, kLongChunks) : std::min(N, kUnits * 2), means = d > kLongRow ? N : 0;
    NormGradLayout l;
    l.partial = (8 * means + 255) / 256 * 256;
    l.total = few_rows(N, d) && d <= kLongRow ? 0 : l.partial + (rows * 2 * d * 4 + 255) / 256 * 256;
    return l;
}

constexpr int64_t kMostRows = INT64_C(1) << 40;

gp_status layer_norm_grad(const void* g, int64_t ldg, gp_dtype grad_dtype, const void* x, int64_t ldx, gp_dtype dtype, int64_t N, int32_t d, const float* stats,
                          const void* weight, gp_dtype weight_dtype, void* x_grad, int64_t ldxg, void* weight_grad, void* bias_grad, int32_t accumulate,
                          void* workspace, int64_t bytes, hipStream_t stream)
{
    if (!known(dtype) || !known(weight_dtype) || !known(grad_dtype))
        return fail(GP_ERR_INVALID_ARG, "unknown dtype %d, %d, %d", (int)dtype, (int)weight_dtype, (int)grad_dtype);
    if (N < 0 || d < 1 || ldx < d || (ldg < d && ldg != 0) || (x_grad && ldxg < d))
        return fail(GP_ERR_INVALID_ARG, "need N >= 0, d >= 1, ldx >= d, ldg >= d or 0, ldxg >= d");
    if (N > kMostRows) return fail(GP_ERR_UNSUPPORTED, "more than 2^40 rows");
    if (N > 0 && (!g || !x || !stats)) return fail(GP_ERR_INVALID_ARG, "NULL argument");
    const bool sums = weight_grad || bias_grad;
    if (!x_grad && !sums) return GP_OK;
    const NormGradLayout l = norm_grad_layout(N, d);
    if (N > 0 && (sums || d > kLongRow) && l.total > 0 && (!workspace || bytes < l.total || (uintptr_t)workspace % 256 != 0))
        return fail(GP_ERR_INVALID_ARG, "need a workspace of %lld bytes on a 256-byte boundary", (long long)l.total);
    NormGradArgs a{};
    a.g = g, a.ldg = ldg, a.x = x, a.ldx = ldx, a.N = N, a.d = d, a.stats = stats, a.weight = weight, a.wide_weights = weight_dtype == GP_F32, a.x_grad = x_grad,
    a.ldxg = ldxg, a.weight_grad = weight_grad, a.bias_grad = bias_grad, a.accumulate = accumulate != 0;
    a.means = (float*)workspace;
    a.partial = sums && l.total > 0 ? (float*)((char*)workspace + l.partial) : nullptr;
    if (N == 0) return accumulate ? GP_OK : launch_join(a, 0, stream);  // (sums of nothing)
    if (dtype == GP_F32) return grad_dtype == GP_F32 ? launch_norm_grad<float, float>(a, stream) : launch_norm_grad<float, bf16_t>(a, stream);
    return grad_dtype == GP_F32 ? launch_norm_grad<bf16_t, float>(a, stream) : launch_norm_grad<bf16_t, bf16_t>(a, stream);
}

}  // namespace

}  // namespace gp

extern "C" gp_status gp_layer_norm(const void* x, int64_t ldx, gp_dtype dtype, int64_t N, int32_t d, const void* weight, const void* bias,
                                   gp_dtype weight_dtype, float eps, void* y, int64_t ldy, gp_dtype out_dtype, float* stats, void* hip_stream)
{
    try {
        return gp::layer_norm(x, ldx, dtype, N, d, weight, bias, weight_dtype, eps, y, ldy, out_dtype, stats, (hipStream_t)hip_stream);
    } catch (const std::exception& e) {
        return gp::fail(GP_ERR_OOM_HOST, "gp_layer_norm: %s", e.what());
    }
}

extern "C" int64_t gp_layer_norm_grad_workspace(int64_t N, int32_t d)
{
    if (N < 0 || N > gp::kMostRows || d < 1) return -1;
    return N == 0 ? 0 : gp::norm_grad_layout(N, d).total;
}

extern "C" gp_status gp_layer_norm_grad(const void* grad, int64_t ldg, gp_dtype grad_dtype, const void* x, int64_t ldx, gp_dtype dtype, int64_t N, int32_t d,
                                        const float* stats, const void* weight, gp_dtype weight_dtype, void* x_grad, int64_t ldxg, void* weight_grad,
                                        void* bias_grad, int32_t accumulate, void* workspace, int64_t workspace_bytes, void* hip_stream)
{
    try {
        return gp::layer_norm_grad(grad, ldg, grad_dtype, x, ldx, dtype, N, d, stats, weight, weight_dtype, x_grad, ldxg, weight_grad, bias_grad, accumulate,
                                   workspace, workspace_bytes, (hipStream_t)hip_stream);
    } catch (const std::exception& e) {
        return gp::fail(GP_ERR_OOM_HOST, "gp_layer_norm_grad: %s", e.what());
    }
}
