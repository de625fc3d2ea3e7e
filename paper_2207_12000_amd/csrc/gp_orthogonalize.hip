// Update directions of weight matrices by Newton-Schulz products, and the step of a weight matrix around them.
//
//     X = U / (|U|_F + eps),   then, step by step,   A = X X^T,   B = b A + c A A,   X <- a X + B X,
//
// X being U or its transpose, whichever has no more rows (m) than columns (n).  Every step maps each singular value s of X to
// a s + b s^3 + c s^5 and leaves the singular vectors alone.  (K. Jordan's Muon optimiser takes such directions from
// the momentum of a weight matrix's gradient.)
//
// Arithmetic.  What the steps leave of a direction that is weak in U is its share times a^steps (485 for five steps of the
// usual a = 3.4445), and so are the roundings on the way: with bf16 operands the result was 1.4e-2 off for normal matrices and
// 0.35 off (relative error in the Frobenius norm) for gradients of low rank over a floor of noise; with single f16
// operands 1.3e-3 and 2.8e-2.  So every matrix is held as two f16 parts, x = hi + lo with 22 bits between them, and a product is three
// f16 products with fp32 accumulation, hi hi + hi lo + lo hi: 3.7e-7 and 9e-6, where fp32 arithmetic itself left 1.6e-6 and
// 1.7e-5.  (Of matrices with a shorter side of up to 16, whose sums have few terms, fp32 left less; where these go in one launch they have
// three parts, TinyParts.)  A singular value after any number of steps is at most what the polynomial makes of [0, 1], and no element exceeds
// the largest singular value: a power of two per matrix and step, known beforehand, keeps every part inside f16's range
// and lo above its subnormal numbers where it counts.
//
// Every product is taken as rows times rows (both operands consecutive along the summed dimension): A and B are symmetric,
// and X is kept in both orientations.  (Iterating on A alone and multiplying X once at the end would take fewer products for long matrices, but
// its roundings grow by a^2 a step: NaN after five on most matrices tried, in 22 bits.)
//
// What bounds it, and us measured (five steps).  Large matrices: power.  The third product of 4096 x 4096 takes 355 us, 1.16 PFLOP/s of f16 products,
// with the matrix cores 60 % busy at 1.9 GHz; the same launch on operands that are all one number takes 210.  The whole, 3.7 - 3.9 ms, of which
// the symmetric products, half of whose tiles are computed, take 198 each; a library's fp32 products take 14.7.  Middle sizes: how evenly tiles fill
// the chip, and the planes' traffic (two 1024 x 4096 steps with bf16 gradients 646: as traced, X X^T 49, whose 72 tiles of 128 by three workgroups each
// leave 40 of 256 compute units idle, A A 21, 272 tiles of 64, the update 66 a step, the start 24, norms and momentum 21).  Small ones: the
// chain of 17 launches, 5 us each, of which a launch on its own would take 1.6 and lines that the launch before has sent past the L2s another 2
// (two 256 x 256 79, 602 x 256 in bf16 92; a barrier among 64 workgroups inside a launch takes 1.4, 2.2 where they hand on what they have by
// device-wide atomics, 20 by fences).  Up to 64 x 256 one launch: 8 (16 x 16), 16 (64 x 64), 24 (256 x 40), 34 (64 x 256); 45 to 62 for
// 256 x 40 in several.
#include <algorithm>
#include <cmath>
#include <exception>
#include <type_traits>

#include "gp_internal.h"

namespace gp {

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;          // sides of planes are multiples of it; what is added is zero
constexpr int kNormBlocks = 256;   // partial sums of squares per matrix
constexpr int kMaxSteps = 32;
constexpr int kMaxShared = 256;     // tiles of a product that several workgroups may share

typedef unsigned short bf16_t;
typedef _Float16 f16;
typedef f16 v4h __attribute__((ext_vector_type(4)));
typedef f16 v8h __attribute__((ext_vector_type(8)));
typedef int v2i __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16_t v) { return __uint_as_float((unsigned)v << 16); }

struct Update {  // U, element by element: G, or the momentum step M <- mu M + G and U = G + mu M (Nesterov) or M
    const void* G;
    int64_t ldg, stride_g;
    const float* M;
    float* M_out;
    int64_t ldm, stride_m;
    float mu;
    int nesterov;
    int64_t rows, cols;
};

// ---- the sum of squares, and the new momentum ---------------------------------------------------------

template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double* part)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < THREADS / 64; ++w) s += part[w];
    return s;
}

// Four neighbours of a row per thread and step, four steps' requests at once (4096 x 4096 fp32: 19 us, 3.5 TB/s; one element at a time
// took 130).  Workgroups of 256 threads where these have no more than one step to do (256 x 256: 3 us, 5 with 1024), else of 1024.
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));
typedef bf16_t v4b_any __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ void load_some(const float* p, int count, float (&v)[4])
{
    if (count >= 4) {
        const v4f_any x = *(const v4f_any*)p;
        v[0] = x[0], v[1] = x[1], v[2] = x[2], v[3] = x[3];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < count ? p[i] : 0.0f;
    }
}
__device__ __forceinline__ void load_some(const bf16_t* p, int count, float (&v)[4])
{
    if (count >= 4) {
        const v4b_any x = *(const v4b_any*)p;
        v[0] = widen(x[0]), v[1] = widen(x[1]), v[2] = widen(x[2]), v[3] = widen(x[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < count ? widen(p[i]) : 0.0f;
    }
}
__device__ __forceinline__ void store_some(float* p, int count, const float (&v)[4])
{
    if (count >= 4) {
        *(v4f_any*)p = (v4f_any){v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < count) p[i] = v[i];
    }
}

template <int kNormThreads, typename T>
__global__ __launch_bounds__(kNormThreads) void gp_ns_norms(Update u, double* __restrict__ partial, int* __restrict__ arrived)
{
    __shared__ double part[kNormThreads / 64];
    if (blockIdx.x == 0 && blockIdx.y == 0)
        for (int i = threadIdx.x; i < kMaxShared; i += kNormThreads) arrived[i] = 0;
    constexpr int U = 4;
    const int64_t z = blockIdx.y, groups = (u.cols + 3) / 4, total = u.rows * groups;
    const T* const G = (const T*)u.G + z * u.stride_g;
    double s = 0.0;
    for (int64_t i = (int64_t)blockIdx.x * kNormThreads + threadIdx.x; i < total; i += (int64_t)U * kNormBlocks * kNormThreads) {
        float g[U][4], m[U][4];
        int64_t at[U];
        int count[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t e = i + (int64_t)k * kNormBlocks * kNormThreads;
            const int64_t r = total <= 0xFFFFFFFFll ? (int64_t)((uint32_t)e / (uint32_t)groups) : e / groups, c = (e - r * groups) * 4;
            count[k] = e < total ? (int)min(u.cols - c, (int64_t)4) : 0;
            at[k] = z * u.stride_m + r * u.ldm + c;
            load_some(G + (count[k] ? r * u.ldg + c : 0), count[k], g[k]);
            if (u.M) load_some(u.M + (count[k] ? at[k] : 0), count[k], m[k]);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (u.M) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    m[k][j] = u.mu * m[k][j] + g[k][j];
                    g[k][j] = u.nesterov ? g[k][j] + u.mu * m[k][j] : m[k][j];
                }
                if (count[k]) store_some(u.M_out + at[k], count[k], m[k]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) s += (double)g[k][j] * g[k][j];
        }
    }
    s = block_sum<kNormThreads>(s, part);
    if (threadIdx.x == 0) partial[z * kNormBlocks + blockIdx.x] = s;
}

// ---- the first X, in two parts and both orientations --------------------------------------------------

__device__ __forceinline__ void split(float v, f16& hi, f16& lo)
{
    // (v as it is rounded to fp32: an instruction that multiplies and rounds to f16 at once can give a neighbour of hi, which
    // the compiler may take for one of hi's two uses alone)
    asm("" : "+v"(v));
    hi = (f16)v;
    lo = (f16)(v - (float)hi);
}

// a third part: what two leave of a number, 33 bits in all
__device__ __forceinline__ void split(float v, f16& hi, f16& lo, f16& rest)
{
    asm("" : "+v"(v));
    split(v, hi, lo);
    rest = (f16)(v - (float)hi - (float)lo);
}

constexpr int kParts = 32;  // from a first part to its second
__device__ __forceinline__ int64_t place(int64_t c) { return (c >> 5) * (2 * kParts) + (c & 31); }

// four neighbours of a plane's row
__device__ __forceinline__ void store_parts(f16* d, const float (&v)[4])
{
    v4h hi, lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f16 x, y;
        split(v[i], x, y);
        hi[i] = x, lo[i] = y;
    }
    *(v4h*)d = hi, *(v4h*)(d + kParts) = lo;
}

// sixteen
__device__ __forceinline__ void store_parts16(f16* d, const float (&v)[16])
{
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        v8h hi, lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f16 x, y;
            split(v[8 * g + i], x, y);
            hi[i] = x, lo[i] = y;
        }
        *(v8h*)(d + 8 * g) = hi, *(v8h*)(d + 8 * g + kParts) = lo;
    }
}

// One 64 x 64 tile per workgroup: a thread loads a square of 4 x 4 elements, whose rows go into one plane and whose columns into the
// other.
template <typename T>
__global__ __launch_bounds__(kThreads) void gp_ns_start(Update u, const double* __restrict__ partial, float eps, float scale, f16* natural,
                                                        f16* transposed, int64_t stride, int ldn, int ldt)
{
    __shared__ double part[kThreads / 64];
    const int64_t z = blockIdx.z;
    const T* const G = (const T*)u.G + z * u.stride_g;
    const int64_t r0 = (int64_t)blockIdx.y * kTile + (threadIdx.x >> 4) * 4, c0 = (int64_t)blockIdx.x * kTile + (threadIdx.x & 15) * 4;
    float v[4][4], m[4][4];
    int count[4];
    const double mine = partial[z * kNormBlocks + threadIdx.x];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t r = r0 + i;
        count[i] = r < u.rows ? (int)max((int64_t)0, min(u.cols - c0, (int64_t)4)) : 0;
        load_some(G + (count[i] ? r * u.ldg + c0 : 0), u.M && !u.nesterov ? 0 : count[i], v[i]);
        if (u.M) load_some(u.M_out + (count[i] ? z * u.stride_m + r * u.ldm + c0 : 0), count[i], m[i]);
    }
    if (u.M)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] = u.nesterov ? v[i][j] + u.mu * m[i][j] : m[i][j];
    static_assert(kNormBlocks == kThreads, "one partial sum per thread");
    const double norm = sqrt(block_sum<kThreads>(mine, part));
    const double factor = (double)scale / (norm + (double)eps);  // (it, or its inverse, may be beyond fp32)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = j < count[i] ? (float)((double)v[i][j] * factor) : 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float t[4] = {v[0][i], v[1][i], v[2][i], v[3][i]};
        store_parts(natural + z * stride + (r0 + i) * ldn + place(c0), v[i]);
        store_parts(transposed + z * stride + (c0 + i) * ldt + place(r0), t);
    }
}

// ---- products ----------------------------------------------------------------------------------------

// D = alpha P Q^T + beta E over planes, D into its own plane and, transposed, into another; or, at the end, into the caller's
// matrix.  A plane's row holds, 32 columns after 32 columns, their first parts and then their second parts (place()): what a step
// of the sum takes of a row is one 128-byte line.
struct Product {
    const f16 *P, *Q, *E;
    int ldp, ldq, lde;   // halves from row to row
    int M, N, K;         // rows of P, rows of Q, summed columns: multiples of 64
    int64_t stride;      // halves from one matrix of the call to the next
    float alpha, beta;
    f16 *D, *Dt;
    int ldd, lddt;
    int symmetric;       // D and Dt are one plane: tiles on and above the diagonal will do
    int tiles_m, tiles_n, tile_count;  // of one matrix
    int64_t all_tiles;   // of all matrices of the call
    int parts;           // workgroups to a tile: each sums over a part of the columns
    float* partial;      // a tile's sums per workgroup
    int* arrived;        // per tile: workgroups whose sums are there (zero between launches)
    // the last product
    int64_t rows, cols;
    void* out;
    int64_t ldo, stride_o;
    const float* W;
    float keep, lr;
};

// all but the wave's last N loads have arrived, it has read what it asked LDS for, and so have the workgroup's others
template <int N>
__device__ __forceinline__ void wait_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

typedef __attribute__((address_space(1))) const void* GlobalPtr;
typedef __attribute__((address_space(3))) void* LdsPtr;

// Tiles of a matrix are numbered in bands of four rows, column by column; where D is symmetric, those on and above the diagonal, a
// band's triangle first.  Each of the chip's eight parts, which share an L2 and take every eighth workgroup, gets one stretch of the
// numbers: a square of tiles, whose lines it reads once.
constexpr int kBand = 4;
int64_t tile_numbers(int64_t tiles_m, int64_t tiles_n, bool symmetric) { return symmetric ? tiles_m * (tiles_m + 1) / 2 : tiles_m * tiles_n; }
__device__ __forceinline__ void tile_at(const Product& a, int t, int& bi, int& bj)
{
    for (int b = 0;; b += kBand) {
        const int rows = min(a.tiles_m - b, kBand), corner = a.symmetric ? rows * (rows + 1) / 2 : 0;
        const int first = a.symmetric ? b + rows : 0, size = corner + rows * (a.tiles_n - first);
        if (t >= size) {
            t -= size;
            continue;
        }
        if (t >= corner) {
            t -= corner;
            bi = b + t % rows, bj = first + t / rows;
            return;
        }
        int c = 0;  // column c of the triangle has c + 1 tiles
        while (t > c) t -= ++c;
        bi = b + t, bj = b + c;
        return;
    }
}
__device__ __forceinline__ int64_t stretched_block() { return (int64_t)(blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3); }
template <typename TO>
__device__ __forceinline__ void store_out(const Product& a, int64_t o, float v)
{
    if constexpr (sizeof(TO) == 4)
        ((float*)a.out)[o] = v;
    else
        ((bf16_t*)a.out)[o] = __builtin_bit_cast(bf16_t, (__bf16)v);
}
template <typename TO>
__device__ __forceinline__ void write_out(const Product& a, int64_t o, float v)
{
    store_out<TO>(a, o, a.W ? a.keep * a.W[o] - a.lr * v : v);
}
// the first `count` of four and of sixteen neighbours of a row, from any element's boundary
template <typename TO>
__device__ __forceinline__ void write_some(const Product& a, int64_t o, int count, const float (&v)[4])
{
    float x[4] = {v[0], v[1], v[2], v[3]};
    if (count <= 0) return;
    if (a.W) {
        float w[4];
        load_some(a.W + o, count, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = a.keep * w[i] - a.lr * v[i];
    }
    if constexpr (sizeof(TO) == 4) {
        store_some((float*)a.out + o, count, x);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < count) store_out<TO>(a, o + i, x[i]);
    }
}
typedef bf16_t v8b_any __attribute__((ext_vector_type(8), aligned(2)));
template <typename TO>
__device__ __forceinline__ void write_row(const Product& a, int64_t o, int count, const float (&v)[16])
{
    if (count < 16) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (i < count) write_out<TO>(a, o + i, v[i]);
        return;
    }
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = v[i];
    if (a.W) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const v4f_any w = *(const v4f_any*)(a.W + o + 4 * g);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * g + i] = a.keep * w[i] - a.lr * v[4 * g + i];
        }
    }
    if constexpr (sizeof(TO) == 4) {
#pragma unroll
        for (int g = 0; g < 4; ++g) *(v4f_any*)((float*)a.out + o + 4 * g) = (v4f_any){x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]};
    } else {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            v8b_any y;
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = __builtin_bit_cast(bf16_t, (__bf16)x[8 * g + i]);
            *(v8b_any*)((bf16_t*)a.out + o + 8 * g) = y;
        }
    }
}

// BM x BN tiles of D by WM x WN waves.  A step sums over 32 columns: BM + BN lines of 128 bytes, which go straight from memory to one of
// STAGES parts of LDS while the matrix cores work on another.  A line's 16-byte pieces lie in LDS in the order
// piece ^ (row / 2 mod 8), with which the 16 lanes that LDS serves together read different banks (no conflicts counted).
// What the shape owes to measurement: large tiles, since every product reads its operands from LDS (us for a 4096 x 4096 update in tiles of 64, 128 and
// 256: 500, 396, 350); loads one at a time among the products (256 x 256 tiles, operands of one number, so that power does not hide it: 232
// us, 270 where a step's loads go out together, and 204 without any).
// A wave's registers hold its BM / WM x BN / WN sums as 32 x 32 blocks: lane l has column l mod 32, rows 8 (i / 4) + 4 (l / 32) + i mod 4.
template <int BM, int BN, int WM, int WN, int STAGES, typename TO, bool LAST>
__global__ __launch_bounds__(64 * WM * WN) void gp_ns_product(Product a)
{
    constexpr int kWaves = WM * WN;
    constexpr int RB = BM / WM / 32, CB = BN / WN / 32;  // blocks of a wave
    constexpr int kLoads = (BM + BN) / 8 / kWaves;       // eight lines per wave and load
    constexpr int kStage = (BM + BN) * 64;
    constexpr int kThreadsHere = 64 * kWaves;
    extern __shared__ __align__(128) f16 lds[];
    __shared__ int arrivals;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int steps = a.K / 32;
    const int wr = wave / WN * (RB * 32), wc = wave % WN * (CB * 32);
    // where this lane reads: line wr + lane mod 32, pieces lane / 32 + 2 s (+ 4: second parts), s = 0, 1
    const int swap = (lane >> 1) & 7;
    const f16* const pl = lds + (wr + (lane & 31)) * 64;
    const f16* const ql = lds + (BM + wc + (lane & 31)) * 64;
    constexpr bool kShared = BM * BN <= 128 * 128;  // (choose_cut)
    const int64_t worker = stretched_block();
    if (worker >= a.all_tiles * a.parts) return;
    const int part = kShared ? (int)(worker / a.all_tiles) : 0;
    const int64_t tile = kShared ? worker - part * a.all_tiles : worker;
    const int k0 = kShared ? (int)((int64_t)steps * part / a.parts) : 0, k1 = kShared ? (int)((int64_t)steps * (part + 1) / a.parts) : steps;
    int bi, bj;
    const int64_t z = tile / a.tile_count;
    tile_at(a, (int)(tile - z * a.tile_count), bi, bj);
    const int64_t base = z * a.stride;
    // lines this lane takes part in loading, the first kLoadsP of P, the others of Q; those past the planes' ends repeat the last one (and
    // are not used)
    constexpr int kLoadsP = BM / 8 / kWaves;
    static_assert(BM % (8 * kWaves) == 0 && BN % (8 * kWaves) == 0, "a load is of one plane");
    const f16 *const p0 = a.P + base + (int64_t)bi * BM * a.ldp, *const q0 = a.Q + base + (int64_t)bj * BN * a.ldq;
    unsigned offset[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
        const int line = (u * kWaves + wave) * 8 + (lane >> 3);
        const unsigned piece = (unsigned)((lane & 7) ^ ((line >> 1) & 7)) * 8;
        offset[u] = piece + (u < kLoadsP ? (unsigned)min(line, a.M - 1 - bi * BM) * (unsigned)a.ldp : (unsigned)min(line - BM, a.N - 1 - bj * BN) * (unsigned)a.ldq);
    }
    auto load = [&](int u, int stage, int step) {
        const f16* const from = (u < kLoadsP ? p0 : q0) + (int64_t)min(step, k1 - 1) * 64;  // (steps past the last are not used)
        __builtin_amdgcn_global_load_lds((GlobalPtr)(from + offset[u]), (LdsPtr)(lds + stage * kStage + (u * kWaves + wave) * 512), 16, 0, 0);
    };
    v16f acc[RB][CB];
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[r][c][i] = 0.0f;
    // half a step's operands: 16 columns of the wave's lines, first and second parts
    struct Half {
        v8h p[2][RB], q[2][CB];
    };
    auto read = [&](Half& f, int stage, int s) {
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const int at = (((lane >> 5) + 2 * s + 4 * part) ^ swap) * 8 + stage * kStage;
#pragma unroll
            for (int r = 0; r < RB; ++r) f.p[part][r] = *(const v8h*)(pl + r * 32 * 64 + at);
#pragma unroll
            for (int c = 0; c < CB; ++c) f.q[part][c] = *(const v8h*)(ql + c * 32 * 64 + at);
        }
        __builtin_amdgcn_sched_barrier(0);  // (the reads go out before the products that they run beside)
    };
    // a half step's products; with them, one at a time (a wave that asks for all of them at once waits for the last before it goes on),
    // the loads of a step into a stage
    auto multiply = [&](const Half& f, auto loads, int stage, int step) {
        constexpr int kProducts = 3 * RB * CB;
#pragma unroll
        for (int x = 0; x < 3; ++x)
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int c = 0; c < CB; ++c) {
                    acc[r][c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.p[x == 0][r], f.q[x == 1][c], acc[r][c], 0, 0, 0);
                    if constexpr (decltype(loads)::value) {
                        const int i = (x * RB + r) * CB + c;
#pragma unroll
                        for (int u = 0; u < kLoads; ++u)
                            if (u >= i * kLoads / kProducts && u < (i + 1) * kLoads / kProducts) {
                                __builtin_amdgcn_sched_barrier(0);
                                load(u, stage, step);
                                __builtin_amdgcn_sched_barrier(0);
                            }
                    }
                }
        __builtin_amdgcn_sched_barrier(0);
    };
    // Every half step's reads run beside the half step before it; a stage is loaded again as soon as all waves have its second
    // half in registers.
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
#pragma unroll
        for (int u = 0; u < kLoads; ++u) load(u, s, k0 + s);
    Half f0, f1;
    wait_and_meet<(STAGES - 1) * kLoads>();
    read(f0, 0, 0);
    int stage = 0;
    for (int k = k0; k < k1; ++k) {
        read(f1, stage, 1);
        multiply(f0, std::false_type{}, 0, 0);
        wait_and_meet<(STAGES - 2) * kLoads>();  // the next step's lines are there
        const int next = stage + 1 == STAGES ? 0 : stage + 1;
        read(f0, next, 0);
        multiply(f1, std::true_type{}, stage, k + STAGES);
        stage = next;
    }
    // The sums, 32 x 32 at a time, turned through LDS so that a lane has 16 neighbours of a row (and, for Dt, of a column): requests
    // of 16 bytes instead of 2.  The stages are free behind this barrier: no load is on its way, and every wave has read its last.
    wait_and_meet<0>();
    if (kShared && a.parts > 1) {
        // Each workgroup of the tile leaves its sums in memory, and whoever comes last adds them up, in the parts' order whoever that is, and
        // goes on.  Nobody waits for another.  (Sums go through memory by device-wide atomic stores and loads, which pass by the L2s that
        // the chip's parts do not share: a fence instead would write back and empty these, 10 to 20 us where all workgroups do it.)
        constexpr int kBlocks = RB * CB, kTogether = 4;  // parts whose sums are on their way
        uint64_t* const sums = (uint64_t*)a.partial + tile * a.parts * (BM * BN / 2) + threadIdx.x;
#pragma unroll
        for (int q = 0; q < 8 * kBlocks; ++q) {
            const v16f& from = acc[q / 8 / CB][q / 8 % CB];
            const v2f x = {from[2 * (q % 8)], from[2 * (q % 8) + 1]};
            __hip_atomic_store(sums + part * (BM * BN / 2) + q * kThreadsHere, __builtin_bit_cast(uint64_t, x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        wait_and_meet<0>();  // (all of the workgroup's stores are done before it counts as arrived)
        if (threadIdx.x == 0) arrivals = __hip_atomic_fetch_add(a.arrived + tile, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
        __syncthreads();
        if (arrivals < a.parts) return;
        if (threadIdx.x == 0) __hip_atomic_store(a.arrived + tile, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
        for (int q = 0; q < 16 * kBlocks; ++q) acc[q / 16 / CB][q / 16 % CB][q % 16] = 0.0f;
        for (int w = 0; w < a.parts; w += kTogether) {
            uint64_t x[kTogether][8 * kBlocks];
#pragma unroll
            for (int t = 0; t < kTogether; ++t)
#pragma unroll
                for (int q = 0; q < 8 * kBlocks; ++q)
                    x[t][q] = __hip_atomic_load(sums + min(w + t, a.parts - 1) * (BM * BN / 2) + q * kThreadsHere, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < kTogether; ++t) {
                if (w + t >= a.parts) break;
#pragma unroll
                for (int q = 0; q < 8 * kBlocks; ++q) {
                    const v2f y = __builtin_bit_cast(v2f, x[t][q]);
                    v16f& to = acc[q / 8 / CB][q / 8 % CB];
                    to[2 * (q % 8)] += y[0], to[2 * (q % 8) + 1] += y[1];
                }
            }
        }
    }
    float* const turn = (float*)lds + wave * (32 * 33);
    const int lr = lane >> 1, lc = (lane & 1) * 16;
    v8h e[2][4];  // of this block and the next: first and second parts of 16 neighbours
    auto fetch = [&](int n) {
        const int r0 = bi * BM + wr + n / CB * 32, c0 = bj * BN + wc + n % CB * 32;
        if (!a.E || r0 >= a.M || c0 >= a.N) return;
        const f16* const p = a.E + base + (int64_t)(r0 + lr) * a.lde + place(c0 + lc);
        e[n & 1][0] = *(const v8h*)p, e[n & 1][1] = *(const v8h*)(p + 8);
        e[n & 1][2] = *(const v8h*)(p + kParts), e[n & 1][3] = *(const v8h*)(p + kParts + 8);
    };
    fetch(0);
#pragma unroll
    for (int n = 0; n < RB * CB; ++n) {
        if (n + 1 < RB * CB) fetch(n + 1);
        const int rb = n / CB, cb = n % CB;
        const int r0 = bi * BM + wr + rb * 32, c0 = bj * BN + wc + cb * 32;
        if (r0 >= a.M || c0 >= a.N) continue;
#pragma unroll
        for (int i = 0; i < 16; ++i) turn[((i >> 2) * 8 + (lane >> 5) * 4 + (i & 3)) * 33 + (lane & 31)] = acc[rb][cb][i];
        __builtin_amdgcn_wave_barrier();
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = turn[lr * 33 + lc + i] * a.alpha;
        if (a.E)
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] += a.beta * ((float)e[n & 1][i >> 3][i & 7] + (float)e[n & 1][2 + (i >> 3)][i & 7]);
        __builtin_amdgcn_wave_barrier();
        if constexpr (LAST) {
            if (r0 + lr >= a.rows) continue;
            write_row<TO>(a, z * a.stride_o + (int64_t)(r0 + lr) * a.ldo + c0 + lc, (int)min(a.cols - c0 - lc, (int64_t)16), v);
        } else {
            store_parts16(a.D + base + (int64_t)(r0 + lr) * a.ldd + place(c0 + lc), v);
            if (a.symmetric && bi == bj) continue;  // (the tile holds both halves)
#pragma unroll
            for (int i = 0; i < 16; ++i) turn[lr * 33 + lc + i] = v[i];
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = turn[(lc + i) * 33 + lr];
            __builtin_amdgcn_wave_barrier();
            store_parts16(a.Dt + base + (int64_t)(c0 + lr) * a.lddt + place(r0 + lc), v);
        }
    }
}

// The same for products of few tiles, where a launch lasts as long as its loads take to arrive: 32 x 32 tiles, the sum's lines dealt out
// to eight wavefronts, which load them straight into the matrix instructions' registers, two lines' worth ahead, and add up
// their sums in LDS.
constexpr int kSmallWaves = 8;

template <typename TO, bool LAST, bool SHARED>
__global__ __launch_bounds__(64 * kSmallWaves) void gp_ns_product_small(Product a)
{
    __shared__ __align__(16) float part[kSmallWaves][32][36];
    [[maybe_unused]] __shared__ int arrivals;
    int bi = blockIdx.y, bj = blockIdx.x;
    if (a.symmetric) {  // rows of the triangle from both ends fill one row of the grid (workgroups that end at once leave units idle: X X^T
        const int n = a.tiles_n, even = n % 2 == 0;  // of 704 x 2000 took 30 us, 17 so, and A A of 704 x 704 12.7, 8.4 so)
        const bool upper = bj >= bi + even;
        bj = upper ? bj - even : n - 1 - bj, bi = upper ? bi : n - even - bi;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int matrix = SHARED ? blockIdx.z / a.parts : blockIdx.z, share = SHARED ? blockIdx.z - matrix * a.parts : 0;  // (of the columns)
    const int64_t base = matrix * a.stride;
    const int r0 = bi * 32, c0 = bj * 32;
    // 16 x 16 x 32 instructions: four lanes read 64 bytes of a row (two lanes and 32 bytes, as the 32 x 32 x 16 ones have it, keep the
    // address unit busy for twice as long)
    const int r16 = lane & 15, kg = lane >> 4;
    const f16* const p = a.P + base + (int64_t)(r0 + r16) * a.ldp + kg * 8;
    const f16* const q = a.Q + base + (int64_t)(c0 + r16) * a.ldq + kg * 8;
    v4f acc[2][2];
#pragma unroll
    for (int x = 0; x < 4; ++x) acc[x / 2][x % 2] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
    const int steps = a.K / 32, begin = SHARED ? steps * share / a.parts : 0, end = SHARED ? steps * (share + 1) / a.parts : steps;
    v8h pv[2][2][2], qv[2][2][2];  // [line][16 rows][part]
    auto load = [&](int b, int step) {
        if (step >= end) return;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                pv[b][h][part] = *(const v8h*)(p + (int64_t)h * 16 * a.ldp + (int64_t)step * 64 + part * kParts);
                qv[b][h][part] = *(const v8h*)(q + (int64_t)h * 16 * a.ldq + (int64_t)step * 64 + part * kParts);
            }
    };
    auto multiply = [&](int b, int step) {
        if (step >= end) return;
#pragma unroll
        for (int x = 0; x < 3; ++x)
#pragma unroll
            for (int h = 0; h < 4; ++h)
                acc[h / 2][h % 2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pv[b][h / 2][x == 0], qv[b][h % 2][x == 1], acc[h / 2][h % 2], 0, 0, 0);
    };
    load(0, begin + wave), load(1, begin + wave + kSmallWaves);
    const bool mine = threadIdx.x < 256;  // four neighbours of a row each, at the end
    const int lr = (threadIdx.x >> 3) & 31, lc = (threadIdx.x & 7) * 4, r = r0 + lr, c = c0 + lc;
    v4h eh = {0, 0, 0, 0}, el = {0, 0, 0, 0};
    if (a.E && mine) {
        const f16* const e = a.E + base + (int64_t)r * a.lde + place(c);
        eh = *(const v4h*)e, el = *(const v4h*)(e + kParts);
    }
    for (int k = begin + wave; k < end; k += 2 * kSmallWaves) {
        multiply(0, k);
        load(0, k + 2 * kSmallWaves);
        multiply(1, k + kSmallWaves);
        load(1, k + 3 * kSmallWaves);
    }
#pragma unroll
    for (int h = 0; h < 4; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[wave][h / 2 * 16 + kg * 4 + i][h % 2 * 16 + r16] = acc[h / 2][h % 2][i];
    __syncthreads();
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (mine) {
#pragma unroll
        for (int w = 0; w < kSmallWaves; ++w) {
            const float4 x = *(const float4*)&part[w][lr][lc];
            v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
        }
    }
    if constexpr (SHARED) {  // handed over as gp_ns_product does it
        constexpr int kTogether = 4;
        const int64_t tile = ((int64_t)matrix * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x;
        uint64_t* const sums = (uint64_t*)a.partial + tile * a.parts * 512 + (threadIdx.x & 255);
        if (mine)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const v2f x = {v[2 * q], v[2 * q + 1]};
                __hip_atomic_store(sums + share * 512 + q * 256, __builtin_bit_cast(uint64_t, x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        wait_and_meet<0>();
        if (threadIdx.x == 0) arrivals = __hip_atomic_fetch_add(a.arrived + tile, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
        __syncthreads();
        if (arrivals < a.parts) return;
        if (threadIdx.x == 0) __hip_atomic_store(a.arrived + tile, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (mine) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = 0.0f;
            for (int w = 0; w < a.parts; w += kTogether) {
                uint64_t x[kTogether][2];
#pragma unroll
                for (int t = 0; t < kTogether; ++t)
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        x[t][q] = __hip_atomic_load(sums + min(w + t, a.parts - 1) * 512 + q * 256, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int t = 0; t < kTogether; ++t) {
                    if (w + t >= a.parts) break;
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const v2f y = __builtin_bit_cast(v2f, x[t][q]);
                        v[2 * q] += y[0], v[2 * q + 1] += y[1];
                    }
                }
            }
        }
    }
    if (mine) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = v[i] * a.alpha + a.beta * ((float)eh[i] + (float)el[i]);
    }
    if constexpr (LAST) {
        if (!mine || r >= a.rows) return;
        write_some<TO>(a, matrix * a.stride_o + (int64_t)r * a.ldo + c, (int)min(a.cols - c, (int64_t)4), v);
    } else {
        if (mine) store_parts(a.D + base + (int64_t)r * a.ldd + place(c), v);
        if (a.symmetric && bi == bj) return;  // (the tile holds both halves)
        __syncthreads();
        if (mine)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[0][lc + i][lr] = v[i];
        __syncthreads();
        if (!mine) return;
        const float4 x = *(const float4*)&part[0][lr][lc];
        const float t[4] = {x.x, x.y, x.z, x.w};
        store_parts(a.Dt + base + (int64_t)(c0 + lr) * a.lddt + place(r0 + lc), t);
    }
}

// A step's second and third product at once, for m <= 128: on 16 columns of X, X <- a X + b Y + c A Y with Y = A X needs no other columns.
// A (in the registers of m / 16 wavefronts, 16 rows each) is read once, X and Y lie in LDS; one launch less per step, where launches are
// what a step takes (us per launch here, and for the two products: 5.6 and 10 with m = 64, 6.5 and 10 with 128, but 12 and 10 with
// 256, where a compute unit reads 256 KB of A).
struct Panel {
    const f16 *A, *Xt;       // planes: m x m, n x m
    f16 *X_out, *Xt_out;     // m x n, n x m
    int m, n;
    int64_t stride;
    float y_scale, fa, fb, fc;
    // the last step
    int64_t rows, cols;
    int tall;
    Product last;
};

template <int M, typename TO, bool LAST>
__global__ __launch_bounds__(4 * M) void gp_ns_panel(Panel a)
{
    constexpr int kSteps = M / 32, kLd = 2 * M + 8;  // halves of a column in LDS: 16 bytes more than its parts, so that columns start on different banks
    __shared__ __align__(16) f16 xs[16 * kLd], ys[16 * kLd];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, kg = lane >> 4;
    const int64_t base = (int64_t)blockIdx.z * a.stride;
    const int c0 = blockIdx.x * 16;
    v8h av[kSteps][2];
    const f16* const arow = a.A + base + (int64_t)(wave * 16 + r16) * (2 * M) + kg * 8;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) av[s][0] = *(const v8h*)(arow + s * 64), av[s][1] = *(const v8h*)(arow + s * 64 + kParts);
    for (int i = threadIdx.x; i < 16 * M / 4; i += 4 * M) {  // (four pieces of eight halves per thread)
        const int col = i / (M / 4), piece = i % (M / 4);
        *(v8h*)(xs + col * kLd + piece * 8) = *(const v8h*)(a.Xt + base + (int64_t)(c0 + col) * (2 * M) + piece * 8);
    }
    __syncthreads();
    auto product = [&](const f16* cols) {
        v4f acc[3] = {{0, 0, 0, 0}, {0, 0, 0, 0}, {0, 0, 0, 0}};
        const f16* const q = cols + r16 * kLd + kg * 8;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const v8h hi = *(const v8h*)(q + s * 64), lo = *(const v8h*)(q + s * 64 + kParts);
            acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(av[s][0], hi, acc[0], 0, 0, 0);
            acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(av[s][1], hi, acc[1], 0, 0, 0);
            acc[2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(av[s][0], lo, acc[2], 0, 0, 0);
        }
        return acc[0] + (acc[1] + acc[2]);
    };
    // the lane's elements: column c0 + r16, rows r .. r + 3
    const int r = wave * 16 + kg * 4, at = r16 * kLd + (int)place(r);
    const v4f y = product(xs);
    const float yv[4] = {y[0] * a.y_scale, y[1] * a.y_scale, y[2] * a.y_scale, y[3] * a.y_scale};
    store_parts(ys + at, yv);
    const v4h xh = *(const v4h*)(xs + at), xl = *(const v4h*)(xs + at + kParts);
    __syncthreads();
    const v4f z = product(ys);
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a.fa * ((float)xh[i] + (float)xl[i]) + (a.fb * y[i] + a.fc * z[i]);
    const int c = c0 + r16;
    if constexpr (LAST) {
        const Product& p = a.last;
        const int64_t o = blockIdx.z * p.stride_o;
        if (a.tall) {  // (the lane's elements are neighbours)
            if (c < p.rows) write_some<TO>(p, o + c * p.ldo + r, (int)min(p.cols - r, (int64_t)4), v);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (r + i < p.rows && c < p.cols) write_out<TO>(p, o + (r + i) * p.ldo + c, v[i]);
        }
    } else {
        store_parts(a.Xt_out + base + (int64_t)c * (2 * M) + place(r), v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f16 hi, lo;
            split(v[i], hi, lo);
            f16* const d = a.X_out + base + (int64_t)(r + i) * (2 * a.n) + place(c);
            d[0] = hi, d[kParts] = lo;
        }
    }
}

// The whole of it for matrices of up to 64 x 256: one workgroup each, one launch.  A wavefront owns 16 columns of X, whose values stay in
// its registers in fp32 from first to last; LDS holds X's parts in rows (for A = X X^T, a 16 x 16 block on or above the diagonal per
// wavefront, and its mirror image) and in columns (for the panel's own Y = A X, then, in the same place, for A Y), and A's parts: 150 of
// the 160 KB.  A step takes 1 to 6 us: three barriers, LDS reads and 18 to 72 products per wavefront, one after the other.  The matrices
// themselves take the rest: an update of 256 x 40 takes 26 us, 43 where a tall matrix's elements, whose neighbours a lane has in a row, are
// asked for and written one by one; of 40 x 256, 27 us.
struct Tiny {
    Update u;
    float eps;
    int steps, tall;
    float scale;                     // of the first X
    float alpha[kMaxSteps];          // A's scale over X's, squared
    float y_scale[kMaxSteps], fa[kMaxSteps], fb[kMaxSteps], fc[kMaxSteps];  // as in Panel
    Product last;
};
constexpr int kTinyRows = 64, kTinyCols = 256;
constexpr int kRowLd = 2 * kTinyCols + 8, kColLd = 2 * kTinyRows + 8;  // halves: rows and columns start on different banks
constexpr size_t kTinyLds = (size_t)(kTinyRows * kRowLd + kTinyCols * kColLd + kTinyRows * kColLd) * 2;

// A shorter side of up to 16 leaves half of LDS free, and there numbers have three parts and products six part products (those of 2^-33 are left
// out): with so few singular values and terms to a sum, what two parts drop does not average out.  Error over that of fp32 steps on the same matrices (geometric mean over 128
// of them, normal ones / of low rank), two parts, three parts: 1 x 16 1.74 / 1.43, 0.82 / 0.78; 4 x 4 1.47 / 1.35, 0.84 / 0.91; 8 x 256 1.21 / 1.18,
// 0.81 / 0.89; 16 x 16 1.07 / 1.07, 0.72 / 0.90; from 24 on two parts are within 1.06 (24 x 24 0.92 / 1.06, 64 x 64 0.69 / 0.93).  us a call of one matrix:
// 8 x 8 7.8, 16 x 256 14.8 (8.9 and 15.4 with 32 rows in two parts).
template <int PARTS>
struct TinyParts {
    // where a column of X or of A, or a row of X, has its third parts, in halves from its first ones
    static constexpr int kColThird = 2 * kParts, kRowThird = kTinyRows / 2 * kRowLd;
    // the parts of four neighbours of a column
    static __device__ __forceinline__ void take(const float (&v)[4], v4h (&h)[PARTS])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f16 hi, lo, rest;
            if constexpr (PARTS == 3)
                split(v[i], hi, lo, rest), h[2][i] = rest;
            else
                split(v[i], hi, lo);
            h[0][i] = hi, h[1][i] = lo;
        }
    }
    static __device__ __forceinline__ void store(f16* d, const v4h (&h)[PARTS])
    {
#pragma unroll
        for (int part = 0; part < PARTS; ++part) *(v4h*)(d + part * kParts) = h[part];
    }
    static __device__ __forceinline__ void store(f16* d, const float (&v)[4])
    {
        v4h h[PARTS];
        take(v, h);
        store(d, h);
    }
    // eight neighbours of a line; third: where its third parts are
    static __device__ __forceinline__ void load(v8h (&x)[PARTS], const f16* p, int third)
    {
        x[0] = *(const v8h*)p, x[1] = *(const v8h*)(p + kParts);
        if constexpr (PARTS == 3) x[2] = *(const v8h*)(p + third);
    }
    static __device__ __forceinline__ void multiply(v4f (&acc)[3], const v8h (&p)[PARTS], const v8h (&q)[PARTS])
    {
        acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[0], q[0], acc[0], 0, 0, 0);
        acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[1], q[0], acc[1], 0, 0, 0);
        acc[2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[0], q[1], acc[2], 0, 0, 0);
        if constexpr (PARTS == 3) {
            acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[2], q[0], acc[1], 0, 0, 0);
            acc[2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[0], q[2], acc[2], 0, 0, 0);
            acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[1], q[1], acc[1], 0, 0, 0);
        }
    }
};

template <int BLOCKS, typename T, typename TO>  // blocks of 16 rows
__global__ __launch_bounds__(1024) void gp_ns_tiny(Tiny a)
{
    extern __shared__ __align__(128) f16 tiny[];
    __shared__ double part[16];
    f16 *const rows = tiny, *const cols = rows + kTinyRows * kRowLd, *const gram = cols + kTinyCols * kColLd;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, kg = lane >> 4;
    const int64_t z = blockIdx.x;
    const int m = (int)(a.tall ? a.u.cols : a.u.rows), n = (int)(a.tall ? a.u.rows : a.u.cols);  // X is m x n
    const int c = wave * 16 + r16;      // the lane's column; its elements v[g][i]: row 16 g + 4 kg + i
    const int panels = (n + 31) / 32 * 2;  // (whole lines of columns)
    const bool active = wave < panels;
    constexpr int kLines = (BLOCKS + 1) / 2, PARTS = BLOCKS == 1 ? 3 : 2;
    using Parts = TinyParts<PARTS>;
    // U, element by element, and the new momentum.  The lane's four elements of a block are neighbours in a tall matrix's rows
    const T* const G = (const T*)a.u.G + z * a.u.stride_g;
    float v[BLOCKS][4], mo[BLOCKS][4];
    double sum = 0.0;
    auto first_row = [&](int g) { return 16 * g + 4 * kg; };
    auto held = [&](int g) { return c < n ? max(0, min(4, m - first_row(g))) : 0; };  // of the four, those that the matrix has
    auto read = [&](const auto* from, int64_t ld, int g, float(&x)[4]) {
        const int count = held(g);
        if (a.tall) {
            load_some(from + (count ? c * ld + first_row(g) : 0), count, x);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = i < count ? widen(from[(first_row(g) + i) * ld + c]) : 0.0f;
        }
    };
    auto write = [&](float* to, int64_t ld, int g, const float(&x)[4]) {
        const int count = held(g);
        if (a.tall) {
            if (count) store_some(to + c * ld + first_row(g), count, x);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < count) to[(first_row(g) + i) * ld + c] = x[i];
        }
    };
#pragma unroll
    for (int g = 0; g < BLOCKS; ++g) read(G, a.u.ldg, g, v[g]);
    if (a.u.M) {
#pragma unroll
        for (int g = 0; g < BLOCKS; ++g) read(a.u.M + z * a.u.stride_m, a.u.ldm, g, mo[g]);
#pragma unroll
        for (int g = 0; g < BLOCKS; ++g) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                mo[g][i] = a.u.mu * mo[g][i] + v[g][i];
                v[g][i] = a.u.nesterov ? v[g][i] + a.u.mu * mo[g][i] : mo[g][i];
            }
            write(a.u.M_out + z * a.u.stride_m, a.u.ldm, g, mo[g]);
        }
    }
#pragma unroll
    for (int g = 0; g < BLOCKS; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += (double)v[g][i] * v[g][i];
    const double factor = (double)a.scale / (sqrt(block_sum<1024>(sum, part)) + (double)a.eps);
#pragma unroll
    for (int g = 0; g < BLOCKS; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[g][i] = 16 * g + 4 * kg + i < m && c < n ? (float)((double)v[g][i] * factor) : 0.0f;
    if constexpr (BLOCKS % 2 == 1) {  // the last line's other half: zero from first to last
        const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (active) Parts::store(cols + c * kColLd + place(16 * BLOCKS + 4 * kg), zero);
        if (threadIdx.x < kTinyRows * 4) Parts::store(gram + threadIdx.x / 4 * kColLd + place(16 * BLOCKS + threadIdx.x % 4 * 4), zero);
    }
    for (int k = 0;; ++k) {
        // X into LDS, both ways
        if (active)
#pragma unroll
            for (int g = 0; g < BLOCKS; ++g) {
                // four rows of this column; and, with the neighbouring lane's, two rows of both columns
                v4h h[PARTS];
                Parts::take(v[g], h);
                Parts::store(cols + c * kColLd + place(16 * g + 4 * kg), h);
                const bool odd = lane & 1;
#pragma unroll
                for (int part = 0; part < PARTS; ++part) {
                    const v2i own = __builtin_bit_cast(v2i, h[part]);  // rows 0 and 1, rows 2 and 3
                    const int other = __builtin_amdgcn_mov_dpp(odd ? own[0] : own[1], 0xB1, 0xF, 0xF, true);  // of the lane beside it, the rows it keeps
                    const unsigned mine = (unsigned)(odd ? own[1] : own[0]);
                    const unsigned left = odd ? (unsigned)other : mine, right = odd ? mine : (unsigned)other;
                    f16* const at = rows + (16 * g + 4 * kg + (odd ? 2 : 0)) * kRowLd + place(c & ~1) + (part == 2 ? Parts::kRowThird : part * kParts);
                    *(unsigned*)at = (left & 0xFFFFu) | right << 16;
                    *(unsigned*)(at + kRowLd) = left >> 16 | (right & 0xFFFF0000u);
                }
            }
        __syncthreads();
        if (wave < BLOCKS * (BLOCKS + 1) / 2) {  // A: a block on or above the diagonal, column by column
            const int bj = wave < 1 ? 0 : wave < 3 ? 1 : wave < 6 ? 2 : 3, bi = wave - bj * (bj + 1) / 2;
            const f16 *const p = rows + (bi * 16 + r16) * kRowLd + kg * 8, *const q = rows + (bj * 16 + r16) * kRowLd + kg * 8;
            v4f acc[3] = {{0, 0, 0, 0}, {0, 0, 0, 0}, {0, 0, 0, 0}};
            for (int s = 0; s < panels / 2; ++s) {
                v8h pv[PARTS], qv[PARTS];
                Parts::load(pv, p + s * 64, Parts::kRowThird);
                Parts::load(qv, q + s * 64, Parts::kRowThird);
                Parts::multiply(acc, pv, qv);
            }
            // element i: row 16 bi + 4 kg + i, column 16 bj + r16; and its mirror image
            const v4f x = acc[0] + (acc[1] + acc[2]);
            const float t[4] = {x[0] * a.alpha[k], x[1] * a.alpha[k], x[2] * a.alpha[k], x[3] * a.alpha[k]};
            v4h h[PARTS];
            Parts::take(t, h);
            Parts::store(gram + (bj * 16 + r16) * kColLd + place(bi * 16 + 4 * kg), h);
            if (bi != bj)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f16* const d = gram + (bi * 16 + 4 * kg + i) * kColLd + place(bj * 16 + r16);
#pragma unroll
                    for (int part = 0; part < PARTS; ++part) d[part * kParts] = h[part][i];
                }
        }
        __syncthreads();
        if (active) {
            constexpr bool kKeep = BLOCKS < 4;  // A in registers, where these hold it
            v8h av[BLOCKS][kLines][PARTS];
#pragma unroll
            for (int g = 0; g < BLOCKS; ++g)
#pragma unroll
                for (int s = 0; s < kLines; ++s)
                    if (kKeep) Parts::load(av[g][s], gram + (16 * g + r16) * kColLd + s * 64 + kg * 8, Parts::kColThird);
            auto product = [&](v4f(&y)[BLOCKS]) {  // A times the wavefront's columns in LDS
                v8h q[kLines][PARTS];
#pragma unroll
                for (int s = 0; s < kLines; ++s) Parts::load(q[s], cols + c * kColLd + s * 64 + kg * 8, Parts::kColThird);
#pragma unroll
                for (int g = 0; g < BLOCKS; ++g) {
                    v4f acc[3] = {{0, 0, 0, 0}, {0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
                    for (int s = 0; s < kLines; ++s) {
                        if (!kKeep) Parts::load(av[g][s], gram + (16 * g + r16) * kColLd + s * 64 + kg * 8, Parts::kColThird);
                        Parts::multiply(acc, av[g][s], q[s]);
                    }
                    y[g] = acc[0] + (acc[1] + acc[2]);
                }
            };
            v4f y[BLOCKS], w[BLOCKS];
            product(y);
#pragma unroll
            for (int g = 0; g < BLOCKS; ++g) {  // (the columns' X is not needed again)
                const float t[4] = {y[g][0] * a.y_scale[k], y[g][1] * a.y_scale[k], y[g][2] * a.y_scale[k], y[g][3] * a.y_scale[k]};
                Parts::store(cols + c * kColLd + place(16 * g + 4 * kg), t);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (a wavefront's own columns: no barrier)
            product(w);
#pragma unroll
            for (int g = 0; g < BLOCKS; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[g][i] = a.fa[k] * v[g][i] + (a.fb[k] * y[g][i] + a.fc[k] * w[g][i]);
        }
        if (k + 1 == a.steps) break;
        __syncthreads();  // (A and X's rows are read to their ends)
    }
    const Product& p = a.last;
    if (p.W) {  // (all requests before the first use)
#pragma unroll
        for (int g = 0; g < BLOCKS; ++g) read(p.W + z * p.stride_o, p.ldo, g, mo[g]);
#pragma unroll
        for (int g = 0; g < BLOCKS; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[g][i] = p.keep * mo[g][i] - p.lr * v[g][i];
    }
#pragma unroll
    for (int g = 0; g < BLOCKS; ++g) {
        if constexpr (sizeof(TO) == 4) {
            write((float*)p.out + z * p.stride_o, p.ldo, g, v[g]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < held(g)) store_out<TO>(p, z * p.stride_o + (a.tall ? c : first_row(g) + i) * p.ldo + (a.tall ? first_row(g) + i : c), v[g][i]);
        }
    }
}

// ---- ranges ------------------------------------------------------------------------------------------

// the largest |a s + b s^3 + c s^5| over 0 <= s <= top
double polynomial_bound(double a, double b, double c, double top)
{
    auto value = [&](double s) { return std::fabs(s * (a + s * s * (b + s * s * c))); };
    double best = value(top);
    double roots[2] = {-1.0, -1.0};  // s^2 where the slope a + 3 b s^2 + 5 c s^4 is zero
    if (c != 0.0) {
        const double disc = 9.0 * b * b - 20.0 * a * c;
        if (disc >= 0.0) roots[0] = (-3.0 * b + std::sqrt(disc)) / (10.0 * c), roots[1] = (-3.0 * b - std::sqrt(disc)) / (10.0 * c);
    } else if (b != 0.0) {
        roots[0] = -a / (3.0 * b);
    }
    for (double r : roots)
        if (r > 0.0 && r < top * top) best = std::max(best, value(std::sqrt(r)));
    return best;
}
// the largest |b t + c t^2| over 0 <= t <= top
double quadratic_bound(double b, double c, double top)
{
    double best = std::fabs(top * (b + top * c));
    if (c != 0.0) {
        const double t = -b / (2.0 * c);
        if (t > 0.0 && t < top) best = std::max(best, std::fabs(t * (b + t * c)));
    }
    return best;
}
// the exponent that brings numbers up to `bound` just under 2^15 (f16 ends at 2^16)
int exponent_for(double bound)
{
    int e = 0;
    (void)std::frexp(bound * 1.01, &e);  // bound * 1.01 <= 2^e; the rest of the factor of two takes the roundings
    return std::min(100, std::max(-100, 15 - e));
}

// ---- the call ----------------------------------------------------------------------------------------

// How a product is cut: tiles of 32 (gp_ns_product_small), 64, 128, 128 x 256, 192 or 256, and how many workgroups sum up a tile of 32 to 128,
// a part of the columns each (larger tiles' sums take longer to hand over than that saves).  The cut of the least time by what
// its parts take, in us as measured: a step of 32 columns where few compute units are at work and where all are (power is what
// the large ones run out of), a tile's end, and for shared tiles the hand-over and its share of every workgroup's.  us a launch,
// model / measured (and workgroups to a tile):
//     m x n, K                    32             64               128         128 x 256     192          256
//    256 x 256, 256            4.9 / 4.9      6.2 / 6.5        11 / 10
//    640 x 640, 640 (A A)      7.5 / 8.0      9.0 / 9.9        15 / 18
//    256 x 4096, X X^T          31 / 30       34 / 35          67 / 67
//    the same, shared         11 / 11 (6)     14 / 13 (8)      25 / 24 (8)
//    704 x 2048, X X^T          17 / 17       14 / 13 (3)      22 / 22 (4)
//    704 x 4096, update                       27 / 26          24 / 24
//   1024 x 1024, 1024           31 / 32       15 / 15          19 / 24                    44 / 48      59 / 79
//   1024 x 4096, X X^T          82            41 / 39          32 / 33 (4)
//   1536 x 1536, X X^T                        24 / 25          24 / 27 (3)
//   2048 x 2048, 2048                         75 / 72          61 / 60                    88 / 87     121 / 138
//   the same, X X^T                           57 / 54          50 / 50                    82 / 78     112 / 131
//   4096 x 4096, 4096                        566 / 500        458 / 396                  387 / 400    345 / 350
//   the same, X X^T                          319 / 275        300 / 259                  196 / 198    273 / 262
//   2 of 1024 x 4096, 1024                    83 / 87          68 / 80       55 / 61      99 / 107     76 / 84
struct Cut {
    int bm, bn;
    int64_t tiles;  // of all matrices
    int parts;
    double us;
};
constexpr int kUnits = 256;  // compute units
Cut choose_cut(int64_t m, int64_t n, int64_t k, bool symmetric, int64_t count)
{
    const int64_t steps = k / 32;
    auto tiles = [&](int64_t bm, int64_t bn) { return tile_numbers((m + bm - 1) / bm, (n + bn - 1) / bn, symmetric) * count; };
    Cut best{32, 32, tiles(32, 32), 1, 1e30};
    const int64_t rounds = (best.tiles + kUnits - 1) / kUnits;  // workgroups that share a compute unit
    if (rounds <= 4) best.us = 2.4 + 0.8 * (double)rounds + (0.02 + 0.195 * (double)rounds) * (double)steps;
    for (int64_t parts = 2; parts * best.tiles <= kUnits && 8 * parts <= steps; ++parts) {
        const double us = 3.2 + 0.215 * (double)((steps + parts - 1) / parts) + 1.5 + 0.18 * (double)parts;
        if (us < best.us) best.parts = (int)parts, best.us = us;
    }
    struct Kind {
        int bm, bn;
        double few, all, finish, hand_over, share;
    };
    static const Kind kinds[] = {{256, 256, 1.4, 2.6, 12.0, 0.0, 0.0}, {192, 192, 1.0, 1.46, 10.0, 0.0, 0.0}, {128, 256, 0.85, 1.4, 10.0, 0.0, 0.0},
                                 {128, 128, 0.48, 0.84, 7.0, 1.5, 1.0}, {64, 64, 0.24, 0.33, 4.2, 1.4, 0.45}};
    for (const Kind& c : kinds) {
        if (symmetric && c.bm != c.bn) continue;
        const int64_t T = tiles(c.bm, c.bn);
        // (beyond one per unit: two workgroups with tiles of 64 share one)
        auto step = [&](int64_t units) {
            return units <= kUnits ? c.few + (c.all - c.few) * (double)units / kUnits : std::min(0.52, 0.35 + 0.0015 * (double)(units - kUnits));
        };
        const int64_t full = c.bm == 64 ? 2 * kUnits : kUnits, rest = T % full;
        double us = (double)(T / full) * ((double)steps * step(full) + c.finish);
        if (rest) us += (double)steps * step(rest) + c.finish;
        if (us < best.us) best = {c.bm, c.bn, T, 1, us};
        if (c.share == 0.0) continue;
        for (int64_t parts = 2; parts * T <= kUnits && 2 * parts <= steps; ++parts) {
            us = (double)((steps + parts - 1) / parts) * step(parts * T) + c.finish + c.hand_over + c.share * (double)parts;
            if (us < best.us) best = {c.bm, c.bn, T, (int)parts, us};
        }
    }
    return best;
}
int64_t cut_bytes(const Cut& c) { return c.parts > 1 ? c.tiles * c.parts * c.bm * c.bn * 4 : 0; }

struct NsLayout {
    int64_t m, n;               // shorter and longer side, of whole tiles
    Cut gram, square, update;   // of a step's three products
    int64_t X[2], Xt[2], A, B;  // planes of a matrix, in halves
    int64_t stride;             // halves
    int64_t arrived, partial, planes, total;  // bytes
};
NsLayout ns_layout(int64_t rows, int64_t cols, int64_t count)
{
    NsLayout l;
    l.m = (std::min(rows, cols) + kTile - 1) / kTile * kTile;
    l.n = (std::max(rows, cols) + kTile - 1) / kTile * kTile;
    l.gram = choose_cut(l.m, l.m, l.n, true, count);
    l.square = choose_cut(l.m, l.m, l.m, true, count);
    l.update = choose_cut(l.m, l.n, l.m, false, count);
    int64_t at = 0;
    for (int i = 0; i < 2; ++i) l.X[i] = at, l.Xt[i] = at + 2 * l.m * l.n, at += 4 * l.m * l.n;
    l.A = at, l.B = at + 2 * l.m * l.m, at += 4 * l.m * l.m;
    l.stride = at;
    l.arrived = (count * kNormBlocks * 8 + 255) / 256 * 256;
    l.partial = l.arrived + kMaxShared * 4;
    l.planes = l.partial + std::max(cut_bytes(l.gram), l.m <= 128 ? 0 : std::max(cut_bytes(l.square), cut_bytes(l.update)));
    l.total = l.planes + count * l.stride * 2;
    return l;
}

bool tiny_shape(int64_t rows, int64_t cols) { return std::min(rows, cols) <= kTinyRows && std::max(rows, cols) <= kTinyCols; }

constexpr int64_t kMaxSide = 1 << 20;
constexpr float kDefaultCoeff[3] = {3.4445f, -4.7750f, 2.0315f};

// what is written: matrices one behind the other, or side by side in rows long enough for all of them
gp_status check_apart(const char* what, int64_t rows, int64_t cols, int64_t count, int64_t ld, int64_t stride)
{
    if (count <= 1 || rows == 0 || cols == 0) return GP_OK;
    if (stride >= (rows - 1) * ld + cols || (stride >= cols && ld >= (count - 1) * stride + cols)) return GP_OK;
    return fail(GP_ERR_INVALID_ARG, "matrices of %s overlap", what);
}

gp_status check_shape(int64_t rows, int64_t cols, int64_t count)
{
    if (rows < 0 || cols < 0 || count < 0) return fail(GP_ERR_INVALID_ARG, "negative size");
    if (rows > kMaxSide || cols > kMaxSide || count > 65535)
        return fail(GP_ERR_UNSUPPORTED, "%lld matrices of %lld x %lld: at most 65535 of 2^20 x 2^20", (long long)count, (long long)rows, (long long)cols);
    return GP_OK;
}

template <int BM, int BN, int WM, int WN, int STAGES, typename TO, bool LAST>
gp_status launch_tiles(const Product& a, hipStream_t stream)
{
    constexpr size_t lds = STAGES * (BM + BN) * 128;
    if constexpr (lds >= 65536) {  // (there are a few bytes of its own beside it)
        gp_status st = raise_lds<&gp_ns_product<BM, BN, WM, WN, STAGES, TO, LAST>>(lds);
        if (st != GP_OK) return st;
    }
    profile_begin("gp_ns_product", stream);
    hipLaunchKernelGGL((gp_ns_product<BM, BN, WM, WN, STAGES, TO, LAST>), dim3((unsigned)((a.all_tiles * a.parts + 7) / 8 * 8)), dim3(64 * WM * WN), lds, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    return GP_OK;
}

template <typename TO, bool LAST>
gp_status launch_product(Product a, const Cut& cut, int64_t count, hipStream_t stream)
{
    // (the last product of a tall matrix is the transpose of the one that the cut was made for)
    const bool turned = a.M != a.N && (a.M > a.N);
    const int bm = turned ? cut.bn : cut.bm, bn = turned ? cut.bm : cut.bn;
    a.tiles_m = (a.M + bm - 1) / bm, a.tiles_n = (a.N + bn - 1) / bn;
    a.tile_count = (int)tile_numbers(a.tiles_m, a.tiles_n, a.symmetric);
    a.all_tiles = a.tile_count * count, a.parts = cut.parts;
    if (bm == 256 && bn == 256) return launch_tiles<256, 256, 2, 2, 2, TO, LAST>(a, stream);
    if (bm == 192) return launch_tiles<192, 192, 2, 2, 3, TO, LAST>(a, stream);
    if (bm == 128 && bn == 256) return launch_tiles<128, 256, 2, 4, 3, TO, LAST>(a, stream);
    if constexpr (LAST)
        if (bm == 256) return launch_tiles<256, 128, 4, 2, 3, TO, LAST>(a, stream);
    if (bm == 128) return launch_tiles<128, 128, 2, 4, 4, TO, LAST>(a, stream);
    if (bm == 64) return launch_tiles<64, 64, 2, 2, 4, TO, LAST>(a, stream);
    profile_begin("gp_ns_product", stream);
    const int even = a.tiles_n % 2 == 0;
    const dim3 grid(a.tiles_n + (a.symmetric ? even : 0), a.symmetric ? (a.tiles_n + 1) / 2 : a.tiles_m, (unsigned)(count * a.parts));
    if constexpr (!LAST)  // (the last product has too few columns for its tiles to be shared)
        if (a.parts > 1) hipLaunchKernelGGL((gp_ns_product_small<TO, false, true>), grid, dim3(64 * kSmallWaves), 0, stream, a);
    if (LAST || a.parts == 1) hipLaunchKernelGGL((gp_ns_product_small<TO, LAST, false>), grid, dim3(64 * kSmallWaves), 0, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    return GP_OK;
}

template <typename TO, bool LAST>
gp_status launch_panels(const Panel& a, int64_t count, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.n / 16), 1, (unsigned)count), block(4 * a.m);
    profile_begin("gp_ns_panel", stream);
    if (a.m == 64)
        hipLaunchKernelGGL((gp_ns_panel<64, TO, LAST>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((gp_ns_panel<128, TO, LAST>), grid, block, 0, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    return GP_OK;
}

template <int BLOCKS, typename T, typename TO>
gp_status launch_tiny(const Tiny& a, int64_t count, hipStream_t stream)
{
    gp_status st = raise_lds<&gp_ns_tiny<BLOCKS, T, TO>>(kTinyLds);
    if (st != GP_OK) return st;
    profile_begin("gp_ns_tiny", stream);
    hipLaunchKernelGGL((gp_ns_tiny<BLOCKS, T, TO>), dim3((unsigned)count), dim3(1024), kTinyLds, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    return GP_OK;
}
template <typename T, typename TO>
gp_status launch_tiny(const Tiny& a, int64_t count, hipStream_t stream)
{
    const int64_t m = std::min(a.u.rows, a.u.cols);
    return m <= 16 ? launch_tiny<1, T, TO>(a, count, stream) : m <= 32 ? launch_tiny<2, T, TO>(a, count, stream) : m <= 48 ? launch_tiny<3, T, TO>(a, count, stream) : launch_tiny<4, T, TO>(a, count, stream);
}

// out: the direction itself (W null, of dtype out_dtype), or the stepped weights
gp_status newton_schulz(const Update& u, gp_dtype dtype, int64_t count, int32_t steps, const float* coeff, float eps, const float* W, float keep,
                        float lr, void* out, int64_t ldo, int64_t stride_o, gp_dtype out_dtype, void* workspace, int64_t bytes, hipStream_t stream)
{
    if (steps < 1 || steps > kMaxSteps) return fail(GP_ERR_INVALID_ARG, "steps = %d: 1 .. %d", steps, kMaxSteps);
    if (!(eps >= 0.0f)) return fail(GP_ERR_INVALID_ARG, "eps must not be negative");
    int ex[kMaxSteps + 1], ea[kMaxSteps], eb[kMaxSteps], ey[kMaxSteps];
    double top = 1.0;
    for (int k = 0; k < steps; ++k) {
        const float* const p = coeff ? coeff + 3 * k : kDefaultCoeff;
        ex[k] = exponent_for(top), ea[k] = exponent_for(top * top), ey[k] = exponent_for(top * top * top), eb[k] = exponent_for(quadratic_bound(p[1], p[2], top * top));
        top = polynomial_bound(p[0], p[1], p[2], top);
        if (!(top <= 1e6)) return fail(GP_ERR_INVALID_ARG, "step %d takes singular values of 0 .. 1 out to %g", k + 1, top);
    }
    if (u.rows == 0 || u.cols == 0 || count == 0) return GP_OK;
    const NsLayout l = ns_layout(u.rows, u.cols, count);
    if (!workspace || bytes < l.total || (uintptr_t)workspace % 256 != 0)
        return fail(GP_ERR_INVALID_ARG, "need a workspace of %lld bytes on a 256-byte boundary", (long long)l.total);
    if (tiny_shape(u.rows, u.cols)) {
        Tiny t{};
        t.u = u, t.eps = eps, t.steps = steps, t.tall = u.rows > u.cols, t.scale = std::ldexp(1.0f, ex[0]);
        for (int k = 0; k < steps; ++k) {
            const float* const p = coeff ? coeff + 3 * k : kDefaultCoeff;
            const int next = k + 1 < steps ? ex[k + 1] : 0;
            t.alpha[k] = std::ldexp(1.0f, ea[k] - 2 * ex[k]), t.y_scale[k] = std::ldexp(1.0f, ey[k] - ea[k] - ex[k]);
            t.fa[k] = std::ldexp(p[0], next - ex[k]), t.fb[k] = std::ldexp(p[1], next - ea[k] - ex[k]), t.fc[k] = std::ldexp(p[2], next - ea[k] - ey[k]);
        }
        t.last.out = out, t.last.ldo = ldo, t.last.stride_o = stride_o, t.last.W = W, t.last.keep = keep, t.last.lr = lr;
        if (dtype == GP_F32) return launch_tiny<float, float>(t, count, stream);
        return out_dtype == GP_F32 ? launch_tiny<bf16_t, float>(t, count, stream) : launch_tiny<bf16_t, bf16_t>(t, count, stream);
    }
    double* const partial = (double*)workspace;
    f16* const ws = (f16*)((char*)workspace + l.planes);
    int* const arrived = (int*)((char*)workspace + l.arrived);
    const bool tall = u.rows > u.cols;

    const dim3 norm_grid(kNormBlocks, (unsigned)count);
    const bool small = u.rows * ((u.cols + 3) / 4) <= 4 * kNormBlocks * kThreads;
    profile_begin("gp_ns_norms", stream);
    if (dtype == GP_F32 && small)
        hipLaunchKernelGGL((gp_ns_norms<kThreads, float>), norm_grid, dim3(kThreads), 0, stream, u, partial, arrived);
    else if (dtype == GP_F32)
        hipLaunchKernelGGL((gp_ns_norms<1024, float>), norm_grid, dim3(1024), 0, stream, u, partial, arrived);
    else if (small)
        hipLaunchKernelGGL((gp_ns_norms<kThreads, bf16_t>), norm_grid, dim3(kThreads), 0, stream, u, partial, arrived);
    else
        hipLaunchKernelGGL((gp_ns_norms<1024, bf16_t>), norm_grid, dim3(1024), 0, stream, u, partial, arrived);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    {
        const int64_t pr = tall ? l.n : l.m, pc = tall ? l.m : l.n;
        const dim3 grid((unsigned)(pc / kTile), (unsigned)(pr / kTile), (unsigned)count);
        f16 *const natural = ws + (tall ? l.Xt[0] : l.X[0]), *const transposed = ws + (tall ? l.X[0] : l.Xt[0]);
        const float scale = std::ldexp(1.0f, ex[0]);
        profile_begin("gp_ns_start", stream);
        if (dtype == GP_F32)
            hipLaunchKernelGGL(gp_ns_start<float>, grid, dim3(kThreads), 0, stream, u, partial, eps, scale, natural, transposed, l.stride, 2 * (int)pc, 2 * (int)pr);
        else
            hipLaunchKernelGGL(gp_ns_start<bf16_t>, grid, dim3(kThreads), 0, stream, u, partial, eps, scale, natural, transposed, l.stride, 2 * (int)pc, 2 * (int)pr);
        profile_end(stream);
        GP_HIP(hipGetLastError());
    }
    const int m = (int)l.m, n = (int)l.n;
    for (int k = 0; k < steps; ++k) {
        const float* const p = coeff ? coeff + 3 * k : kDefaultCoeff;
        f16 *const X = ws + l.X[k & 1], *const Xt = ws + l.Xt[k & 1], *const A = ws + l.A, *const B = ws + l.B;
        Product a{};
        a.stride = l.stride, a.arrived = arrived, a.partial = (float*)((char*)workspace + l.partial);
        a.P = a.Q = X, a.ldp = a.ldq = 2 * n, a.M = a.N = m, a.K = n;
        a.alpha = std::ldexp(1.0f, ea[k] - 2 * ex[k]);
        a.D = a.Dt = A, a.ldd = a.lddt = 2 * m, a.symmetric = 1;
        gp_status st = launch_product<float, false>(a, l.gram, count, stream);
        if (st != GP_OK) return st;
        const bool last_step = k == steps - 1;
        if (m <= 128) {
            Panel q{};
            const int out_ex = last_step ? 0 : ex[k + 1];
            q.A = A, q.Xt = Xt, q.X_out = ws + l.X[(k + 1) & 1], q.Xt_out = ws + l.Xt[(k + 1) & 1];
            q.m = m, q.n = n, q.stride = l.stride, q.tall = tall;
            q.y_scale = std::ldexp(1.0f, ey[k] - ea[k] - ex[k]);
            q.fa = std::ldexp(p[0], out_ex - ex[k]), q.fb = std::ldexp(p[1], out_ex - ea[k] - ex[k]), q.fc = std::ldexp(p[2], out_ex - ea[k] - ey[k]);
            q.last.rows = u.rows, q.last.cols = u.cols, q.last.out = out, q.last.ldo = ldo, q.last.stride_o = stride_o;
            q.last.W = W, q.last.keep = keep, q.last.lr = lr;
            st = !last_step ? launch_panels<float, false>(q, count, stream) : out_dtype == GP_F32 ? launch_panels<float, true>(q, count, stream) : launch_panels<bf16_t, true>(q, count, stream);
            if (st != GP_OK) return st;
            continue;
        }
        a.P = a.Q = a.E = A, a.ldp = a.ldq = a.lde = 2 * m, a.K = m;
        a.alpha = std::ldexp(p[2], eb[k] - 2 * ea[k]), a.beta = std::ldexp(p[1], eb[k] - ea[k]);
        a.D = a.Dt = B;
        if ((st = launch_product<float, false>(a, l.square, count, stream)) != GP_OK) return st;
        a.symmetric = 0;
        if (!last_step) {
            const int next = ex[k + 1] - ex[k];
            a.P = B, a.Q = Xt, a.N = n, a.E = X, a.lde = 2 * n;
            a.alpha = std::ldexp(1.0f, next - eb[k]), a.beta = std::ldexp(p[0], next);
            a.D = ws + l.X[(k + 1) & 1], a.ldd = 2 * n, a.Dt = ws + l.Xt[(k + 1) & 1], a.lddt = 2 * m;
            if ((st = launch_product<float, false>(a, l.update, count, stream)) != GP_OK) return st;
        } else {  // in the orientation of the caller's matrix
            a.P = tall ? Xt : B, a.Q = tall ? B : Xt, a.M = tall ? n : m, a.N = tall ? m : n;
            a.E = tall ? Xt : X, a.lde = tall ? 2 * m : 2 * n;
            a.alpha = std::ldexp(1.0f, -ex[k] - eb[k]), a.beta = std::ldexp(p[0], -ex[k]);
            a.rows = u.rows, a.cols = u.cols, a.out = out, a.ldo = ldo, a.stride_o = stride_o, a.W = W, a.keep = keep, a.lr = lr;
            st = out_dtype == GP_F32 ? launch_product<float, true>(a, l.update, count, stream) : launch_product<bf16_t, true>(a, l.update, count, stream);
            if (st != GP_OK) return st;
        }
    }
    return GP_OK;
}

}  // namespace

}  // namespace gp

extern "C" int64_t gp_orthogonalize_workspace(int64_t rows, int64_t cols, int64_t count)
{
    if (rows < 0 || cols < 0 || count < 0 || rows > gp::kMaxSide || cols > gp::kMaxSide || count > 65535) return -1;
    return rows == 0 || cols == 0 || count == 0 ? 0 : gp::ns_layout(rows, cols, count).total;
}

extern "C" gp_status gp_orthogonalize(const void* G, int64_t ldg, int64_t stride_g, gp_dtype dtype, int64_t rows, int64_t cols, int64_t count,
                                      int32_t steps, const float* coeff, float eps, void* out, int64_t ldo, int64_t stride_o, void* workspace,
                                      int64_t workspace_bytes, void* hip_stream)
{
    using namespace gp;
    try {
        if (dtype != GP_F32 && dtype != GP_BF16) return fail(GP_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
        gp_status st = check_shape(rows, cols, count);
        if (st != GP_OK) return st;
        if (ldg < cols || ldo < cols) return fail(GP_ERR_INVALID_ARG, "need ldg >= cols, ldo >= cols");
        if ((st = check_apart("out", rows, cols, count, ldo, stride_o)) != GP_OK) return st;
        if ((!G || !out) && rows > 0 && cols > 0 && count > 0) return fail(GP_ERR_INVALID_ARG, "NULL argument");
        Update u{};
        u.G = G, u.ldg = ldg, u.stride_g = stride_g, u.rows = rows, u.cols = cols;
        return newton_schulz(u, dtype, count, steps, coeff, eps, nullptr, 0.0f, 0.0f, out, ldo, stride_o, dtype, workspace, workspace_bytes,
                             (hipStream_t)hip_stream);
    } catch (const std::exception& e) {
        return fail(GP_ERR_OOM_HOST, "gp_orthogonalize: %s", e.what());
    }
}

extern "C" gp_status gp_muon_step(const float* W, float* W_out, int64_t ldw, int64_t stride_w, const float* M, float* M_out, int64_t ldm,
                                  int64_t stride_m, const void* G, int64_t ldg, int64_t stride_g, gp_dtype dtype, int64_t rows, int64_t cols,
                                  int64_t count, float lr, float momentum, float weight_decay, int32_t nesterov, int32_t steps,
                                  const float* coeff, float eps, void* workspace, int64_t workspace_bytes, void* hip_stream)
{
    using namespace gp;
    try {
        if (dtype != GP_F32 && dtype != GP_BF16) return fail(GP_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
        gp_status st = check_shape(rows, cols, count);
        if (st != GP_OK) return st;
        if (ldg < cols || ldw < cols || ldm < cols) return fail(GP_ERR_INVALID_ARG, "need ldg >= cols, ldw >= cols, ldm >= cols");
        if ((st = check_apart("W", rows, cols, count, ldw, stride_w)) != GP_OK) return st;
        if ((st = check_apart("M", rows, cols, count, ldm, stride_m)) != GP_OK) return st;
        if ((!G || !W || !W_out || !M || !M_out) && rows > 0 && cols > 0 && count > 0) return fail(GP_ERR_INVALID_ARG, "NULL argument");
        Update u{};
        u.G = G, u.ldg = ldg, u.stride_g = stride_g, u.rows = rows, u.cols = cols;
        u.M = M, u.M_out = M_out, u.ldm = ldm, u.stride_m = stride_m, u.mu = momentum, u.nesterov = nesterov != 0;
        return newton_schulz(u, dtype, count, steps, coeff, eps, W, (float)(1.0 - (double)lr * (double)weight_decay), lr, W_out, ldw, stride_w,
                             GP_F32, workspace, workspace_bytes, (hipStream_t)hip_stream);
    } catch (const std::exception& e) {
        return fail(GP_ERR_OOM_HOST, "gp_muon_step: %s", e.what());
    }
}
