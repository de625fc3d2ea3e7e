// Embedding rows of a model over the hop stack, and their gradient.
//
//   lookup    out[i, :]  = scale * table[token[i], :]                      (zero where the token names no row)
//   gradient  grad[v, :] = scale * sum_{i: token[i] = v} up[i, :]
//
// The gradient is taken by sorted tokens: (token, position) pairs are sorted, which puts the positions of one token next to
// one another in ascending order, and the rows of up are summed along that list.  The list is cut into tiles of equal
// length whatever the tokens are, so a token that half of the positions name costs no more than any other; a token's
// run that a tile boundary cuts leaves one partial row in every tile it touches, and a second launch adds these up in
// tile order.  No atomics: the same inputs give the same bits.  Sums are held in fp32 and rounded once.
#include <algorithm>
#include <type_traits>

#include "gp_internal.h"

namespace gp {

namespace {

constexpr int kThreads = 256;

typedef unsigned short bf16_t;

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16_t v) { return __uint_as_float((unsigned)v << 16); }
template <typename T>
__device__ __forceinline__ T narrow(float v)
{
    if constexpr (std::is_same<T, float>::value)
        return v;
    else
        return __builtin_bit_cast(bf16_t, (__bf16)v);  // to nearest even
}

// N elements from or to any element's boundary: gfx950 loads and stores vectors from there in one request
template <typename T, int N>
struct Vec {
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <typename T, int N>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[N])
{
    if constexpr (N == 1) {
        v[0] = widen(*p);
    } else {
        const typename Vec<T, N>::type x = *reinterpret_cast<const typename Vec<T, N>::type*>(p);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = widen(x[i]);
    }
}
template <typename T, int N>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[N])
{
    if constexpr (N == 1) {
        *p = narrow<T>(v[0]);
    } else {
        typename Vec<T, N>::type x;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = narrow<T>(v[i]);
        *reinterpret_cast<typename Vec<T, N>::type*>(p) = x;
    }
}

// ---- lookup -----------------------------------------------------------------------------------------

struct LookupArgs {
    const void* table;
    int64_t ldt, V;
    int d, nvec;
    const void* tokens;
    int wide;  // tokens are 64 bits each
    int64_t N;
    float scale;
    void* out;
    int64_t ldo;
};

__device__ __forceinline__ int64_t token_at(const void* tokens, int wide, int64_t i)
{
    return wide ? ((const int64_t*)tokens)[i] : (int64_t)((const int32_t*)tokens)[i];
}

// One vector per thread and step, four steps' requests at once.  A row's last vector is moved back to end with the row (what
// it repeats is written twice, identically).
template <typename TI, typename TO, int VEC>
__global__ __launch_bounds__(kThreads) void gp_embedding_rows(LookupArgs a)
{
    constexpr int U = 4;
    const int64_t total = a.N * a.nvec;
    for (int64_t b0 = (int64_t)blockIdx.x * (U * kThreads); b0 < total; b0 += (int64_t)gridDim.x * (U * kThreads)) {
        const int64_t r0 = b0 / a.nvec;
        const unsigned rem = (unsigned)(b0 - r0 * a.nvec);
        int64_t row[U], tok[U];
        int col[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const unsigned x = rem + u * kThreads + threadIdx.x, q = x / (unsigned)a.nvec;
            row[u] = r0 + q;
            col[u] = min((int)(x - q * a.nvec) * VEC, a.d - VEC);
            tok[u] = row[u] < a.N ? token_at(a.tokens, a.wide, row[u]) : -1;
        }
        float v[U][VEC];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[u][i] = 0.0f;
            if (tok[u] >= 0 && tok[u] < a.V) load_vec<TI, VEC>((const TI*)a.table + tok[u] * a.ldt + col[u], v[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (row[u] >= a.N) continue;
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[u][i] *= a.scale;
            if (tok[u] < 0 || tok[u] >= a.V)  // (zero whatever the scale is)
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[u][i] = 0.0f;
            store_vec<TO, VEC>((TO*)a.out + row[u] * a.ldo + col[u], v[u]);
        }
    }
}

template <typename TI, typename TO, int VEC>
gp_status launch_lookup(LookupArgs a, hipStream_t stream)
{
    a.nvec = (a.d + VEC - 1) / VEC;
    const int64_t blocks = (a.N * a.nvec + 4 * kThreads - 1) / (4 * kThreads);
    profile_begin("gp_embedding_rows", stream);
    hipLaunchKernelGGL((gp_embedding_rows<TI, TO, VEC>), dim3((unsigned)std::min<int64_t>(blocks, 1 << 30)), dim3(kThreads), 0, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    return GP_OK;
}
template <typename TI, typename TO>
gp_status launch_lookup(const LookupArgs& a, hipStream_t stream)
{
    constexpr int VEC = sizeof(TI) == 2 && sizeof(TO) == 2 ? 8 : 4;  // 16 bytes of the wider type
    return a.d >= VEC ? launch_lookup<TI, TO, VEC>(a, stream) : launch_lookup<TI, TO, 1>(a, stream);
}

// ---- gradient -----------------------------------------------------------------------------------------

// a sorted list's entry: token << 32 | position; a token that names no row counts as V, behind all that do
__global__ __launch_bounds__(kThreads) void gp_token_keys(const void* __restrict__ tokens, int wide, int64_t N, int64_t V, uint64_t* __restrict__ keys)
{
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < N; i += (int64_t)gridDim.x * kThreads) {
        const int64_t t = token_at(tokens, wide, i);
        keys[i] = (uint64_t)(t >= 0 && t < V ? t : V) << 32 | (uint64_t)i;
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void gp_zero_rows(T* __restrict__ p, int64_t ld, int64_t rows, int d)
{
    const int64_t total = rows * d;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
        const int64_t r = i / d;
        p[r * ld + (i - r * d)] = 0;
    }
}

struct GradArgs {
    const uint64_t* keys;  // sorted
    int64_t N, V, tile, tiles;
    const void* up;
    int64_t ldg;
    int d, nvec;
    float scale;
    void* out;
    int64_t ldt;
    int accumulate;
    float* carry;  // two partial rows of nvec vectors per tile: of the run that came in, of the run that goes on
};

// the finished sums of one vector of one row
template <typename TO, int VEC>
__device__ __forceinline__ void finish(const GradArgs& a, int64_t v, int c, const float (&acc)[VEC])
{
    const int col = min(c * VEC, a.d - VEC);
    TO* p = (TO*)a.out + v * a.ldt + col;
    float r[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) r[i] = acc[i] * a.scale;
    if (!a.accumulate) {
        store_vec<TO, VEC>(p, r);
    } else if (col == c * VEC) {
        float old[VEC];
        load_vec<TO, VEC>(p, old);
#pragma unroll
        for (int i = 0; i < VEC; ++i) r[i] += old[i];
        store_vec<TO, VEC>(p, r);
    } else {  // a last vector that was moved back: what it repeats is added by its neighbour
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (col + i >= c * VEC) p[i] = narrow<TO>(widen(p[i]) + r[i]);
    }
}

// G lanes walk one tile; a lane holds one vector of the sums.
template <typename TG, typename TO, int VEC, int G>
__global__ __launch_bounds__(kThreads) void gp_sum_tiles(GradArgs a)
{
    constexpr int U = 8;
    const int64_t t = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
    const int c = blockIdx.y * G + threadIdx.x % G;
    if (t >= a.tiles || c >= a.nvec) return;
    const int64_t lo = t * a.tile, hi = min(lo + a.tile, a.N);
    const TG* const up = (const TG*)a.up + min(c * VEC, a.d - VEC);
    int64_t cur = (int64_t)(a.keys[lo] >> 32);
    bool came_in = lo > 0 && (int64_t)(a.keys[lo - 1] >> 32) == cur;
    float acc[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = 0.0f;
    for (int64_t p = lo; p < hi; p += U) {
        uint64_t key[U];
        float v[U][VEC];
#pragma unroll
        for (int u = 0; u < U; ++u) key[u] = p + u < hi ? a.keys[p + u] : ~UINT64_C(0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[u][i] = 0.0f;
            if ((int64_t)(key[u] >> 32) < a.V) load_vec<TG, VEC>(up + (int64_t)(key[u] & 0xFFFFFFFFu) * a.ldg, v[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u >= hi) break;
            const int64_t tok = (int64_t)(key[u] >> 32);
            if (tok != cur) {  // (cur < tok <= V)
                if (came_in)
                    store_vec<float, VEC>(a.carry + ((2 * t) * a.nvec + c) * VEC, acc);
                else
                    finish<TO, VEC>(a, cur, c, acc);
                cur = tok, came_in = false;
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < VEC; ++i) acc[i] += v[u][i];
        }
    }
    if (cur >= a.V) return;
    if (came_in)
        store_vec<float, VEC>(a.carry + ((2 * t) * a.nvec + c) * VEC, acc);
    else if (hi < a.N && (int64_t)(a.keys[hi] >> 32) == cur)
        store_vec<float, VEC>(a.carry + ((2 * t + 1) * a.nvec + c) * VEC, acc);
    else
        finish<TO, VEC>(a, cur, c, acc);
}

// One workgroup per tile in which a run begins that goes on: its partial rows, added up in the order of (tile mod groups,
// tile), then over the groups.
template <typename TO, int VEC, int G>
__global__ __launch_bounds__(kThreads) void gp_join_tiles(GradArgs a)
{
    constexpr int kGroups = kThreads / G;
    __shared__ float part[kThreads][VEC];
    const int64_t t = blockIdx.x;
    const int64_t lo = t * a.tile, hi = min(lo + a.tile, a.N);
    const int64_t tok = (int64_t)(a.keys[hi - 1] >> 32);
    if (tok >= a.V || hi >= a.N || (int64_t)(a.keys[hi] >> 32) != tok) return;                   // nothing goes on
    if (lo > 0 && (int64_t)(a.keys[lo - 1] >> 32) == tok) return;                                // it began before
    int64_t first = t + 1, last = a.tiles;  // the first tile whose list does not start with the token: between these
    while (first < last) {
        const int64_t mid = (first + last) / 2;
        if ((int64_t)(a.keys[mid * a.tile] >> 32) == tok) first = mid + 1;
        else last = mid;
    }
    const int g = threadIdx.x / G, c = blockIdx.y * G + threadIdx.x % G;
    float acc[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = 0.0f;
    if (c < a.nvec) {
        if (g == 0) load_vec<float, VEC>(a.carry + ((2 * t + 1) * a.nvec + c) * VEC, acc);
        for (int64_t s = t + 1 + g; s < last; s += kGroups) {
            float v[VEC];
            load_vec<float, VEC>(a.carry + ((2 * s) * a.nvec + c) * VEC, v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) acc[i] += v[i];
        }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) part[threadIdx.x][i] = acc[i];
    __syncthreads();
    if (g > 0 || c >= a.nvec) return;
    for (int o = 1; o < kGroups; ++o)
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] += part[o * G + threadIdx.x][i];
    finish<TO, VEC>(a, tok, c, acc);
}

template <typename TG, typename TO, int VEC, int G>
gp_status launch_sums(const GradArgs& a, hipStream_t stream)
{
    const unsigned ny = (unsigned)((a.nvec + G - 1) / G);
    constexpr int per = kThreads / G;
    profile_begin("gp_sum_tiles", stream);
    hipLaunchKernelGGL((gp_sum_tiles<TG, TO, VEC, G>), dim3((unsigned)((a.tiles + per - 1) / per), ny), dim3(kThreads), 0, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    if (a.tiles > 1) {
        profile_begin("gp_join_tiles", stream);
        hipLaunchKernelGGL((gp_join_tiles<TO, VEC, G>), dim3((unsigned)a.tiles, ny), dim3(kThreads), 0, stream, a);
        profile_end(stream);
        GP_HIP(hipGetLastError());
    }
    return GP_OK;
}
template <typename TG, typename TO, int VEC>
gp_status launch_sums(GradArgs a, hipStream_t stream)
{
    a.nvec = (a.d + VEC - 1) / VEC;
    if (a.nvec <= 8) return launch_sums<TG, TO, VEC, 8>(a, stream);
    if (a.nvec <= 16) return launch_sums<TG, TO, VEC, 16>(a, stream);
    if (a.nvec <= 32) return launch_sums<TG, TO, VEC, 32>(a, stream);
    return launch_sums<TG, TO, VEC, 64>(a, stream);
}
template <typename TG, typename TO>
gp_status launch_sums(const GradArgs& a, hipStream_t stream)
{
    constexpr int VEC = sizeof(TG) == 2 ? 8 : 4;
    return a.d >= VEC ? launch_sums<TG, TO, VEC>(a, stream) : launch_sums<TG, TO, 1>(a, stream);
}

// Tiles: equal lengths; enough of them to fill the chip, few enough that the partial rows of one token are added up fast.
constexpr int64_t kMinTile = 16, kMaxTiles = 16384;
int64_t tile_length(int64_t N) { return std::max(kMinTile, (N + kMaxTiles - 1) / kMaxTiles); }

int bits_of(int64_t v)
{
    int b = 0;
    while (v >> b) ++b;
    return b;
}

struct GradLayout {
    int64_t other, scratch, carry, total;
};
GradLayout grad_layout(int64_t N, int32_t d)
{
    auto up = [](int64_t b) { return (b + 255) / 256 * 256; };
    const int64_t tiles = (N + tile_length(N) - 1) / tile_length(N);
    GradLayout l;
    l.other = up(8 * N);
    l.scratch = l.other + up(8 * N);
    l.carry = l.scratch + up((int64_t)device_sort_scratch_words(N) * 4);
    l.total = l.carry + up(2 * tiles * (((int64_t)d + 7) / 8 * 8) * 4);
    return l;
}

constexpr int64_t kMaxCount = (INT64_C(1) << 31) - 1;

gp_status embedding(const void* table, int64_t ldt, gp_dtype dtype, int64_t V, int32_t d, const void* tokens, gp_index index, int64_t N,
                    float scale, void* out, int64_t ldo, gp_dtype out_dtype, hipStream_t stream)
{
    if ((dtype != GP_F32 && dtype != GP_BF16) || (out_dtype != GP_F32 && out_dtype != GP_BF16))
        return fail(GP_ERR_INVALID_ARG, "unknown dtype %d, %d", (int)dtype, (int)out_dtype);
    if (index != GP_I32 && index != GP_I64) return fail(GP_ERR_INVALID_ARG, "unknown index type %d", (int)index);
    if (N < 0 || V < 1 || d < 1 || ldt < d || ldo < d) return fail(GP_ERR_INVALID_ARG, "need N >= 0, V >= 1, d >= 1, ldt >= d, ldo >= d");
    if (N == 0) return GP_OK;
    if (!table || !tokens || !out) return fail(GP_ERR_INVALID_ARG, "NULL argument");
    if (N > (INT64_C(1) << 62) / std::max(d, 1)) return fail(GP_ERR_OVERFLOW, "N x d does not fit 62 bits");
    LookupArgs a{};
    a.table = table, a.ldt = ldt, a.V = V, a.d = d, a.tokens = tokens, a.wide = index == GP_I64, a.N = N, a.scale = scale, a.out = out,
    a.ldo = ldo;
    if (dtype == GP_F32) return out_dtype == GP_F32 ? launch_lookup<float, float>(a, stream) : launch_lookup<float, bf16_t>(a, stream);
    return out_dtype == GP_F32 ? launch_lookup<bf16_t, float>(a, stream) : launch_lookup<bf16_t, bf16_t>(a, stream);
}

gp_status embedding_grad(const void* tokens, gp_index index, int64_t N, const void* up, int64_t ldg, gp_dtype dtype, int32_t d, float scale,
                         int64_t V, void* out, int64_t ldt, gp_dtype out_dtype, int32_t accumulate, void* workspace, int64_t bytes,
                         hipStream_t stream)
{
    if ((dtype != GP_F32 && dtype != GP_BF16) || (out_dtype != GP_F32 && out_dtype != GP_BF16))
        return fail(GP_ERR_INVALID_ARG, "unknown dtype %d, %d", (int)dtype, (int)out_dtype);
    if (index != GP_I32 && index != GP_I64) return fail(GP_ERR_INVALID_ARG, "unknown index type %d", (int)index);
    if (N < 0 || V < 1 || d < 1 || ldg < d || ldt < d) return fail(GP_ERR_INVALID_ARG, "need N >= 0, V >= 1, d >= 1, ldg >= d, ldt >= d");
    if (N > kMaxCount || V > kMaxCount) return fail(GP_ERR_UNSUPPORTED, "more than 2^31 - 1 tokens or rows");
    if (!out || (N > 0 && (!tokens || !up))) return fail(GP_ERR_INVALID_ARG, "NULL argument");
    const GradLayout l = grad_layout(N, d);
    if (N > 0 && (!workspace || bytes < l.total || (uintptr_t)workspace % 256 != 0))
        return fail(GP_ERR_INVALID_ARG, "need a workspace of %lld bytes on a 256-byte boundary", (long long)l.total);
    if (!accumulate) {
        const unsigned grid = (unsigned)std::min<int64_t>((V * d + kThreads - 1) / kThreads, 256 * 16);
        profile_begin("gp_zero_rows", stream);
        if (out_dtype == GP_F32)
            hipLaunchKernelGGL(gp_zero_rows<float>, dim3(grid), dim3(kThreads), 0, stream, (float*)out, ldt, V, d);
        else
            hipLaunchKernelGGL(gp_zero_rows<bf16_t>, dim3(grid), dim3(kThreads), 0, stream, (bf16_t*)out, ldt, V, d);
        profile_end(stream);
        GP_HIP(hipGetLastError());
    }
    if (N == 0) return GP_OK;
    char* const ws = (char*)workspace;
    uint64_t* const keys = (uint64_t*)ws;
    profile_begin("gp_token_keys", stream);
    hipLaunchKernelGGL(gp_token_keys, dim3((unsigned)std::min<int64_t>((N + kThreads - 1) / kThreads, 256 * 16)), dim3(kThreads), 0, stream, tokens,
                       (int)(index == GP_I64), N, V, keys);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    uint64_t* sorted = nullptr;
    gp_status st = device_sort_keys(keys, (uint64_t*)(ws + l.other), N, 0, bits_of(V), (uint32_t*)(ws + l.scratch), stream, &sorted);
    if (st != GP_OK) return st;
    GradArgs a{};
    a.keys = sorted, a.N = N, a.V = V, a.tile = tile_length(N), a.tiles = (N + a.tile - 1) / a.tile, a.up = up, a.ldg = ldg, a.d = d,
    a.scale = scale, a.out = out, a.ldt = ldt, a.accumulate = accumulate != 0, a.carry = (float*)(ws + l.carry);
    if (dtype == GP_F32) return out_dtype == GP_F32 ? launch_sums<float, float>(a, stream) : launch_sums<float, bf16_t>(a, stream);
    return out_dtype == GP_F32 ? launch_sums<bf16_t, float>(a, stream) : launch_sums<bf16_t, bf16_t>(a, stream);
}

}  // namespace

}  // namespace gp

extern "C" gp_status gp_embedding(const void* table, int64_t ldt, gp_dtype dtype, int64_t V, int32_t d, const void* tokens, gp_index index,
                                  int64_t N, float scale, void* out, int64_t ldo, gp_dtype out_dtype, void* hip_stream)
{
    return gp::embedding(table, ldt, dtype, V, d, tokens, index, N, scale, out, ldo, out_dtype, (hipStream_t)hip_stream);
}

extern "C" int64_t gp_embedding_grad_workspace(int64_t N, int64_t V, int32_t d)
{
    if (N < 0 || N > gp::kMaxCount || V < 1 || V > gp::kMaxCount || d < 1) return -1;
    return N == 0 ? 0 : gp::grad_layout(N, d).total;
}

extern "C" gp_status gp_embedding_grad(const void* tokens, gp_index index, int64_t N, const void* grad, int64_t ldg, gp_dtype dtype, int32_t d,
                                       float scale, int64_t V, void* table_grad, int64_t ldt, gp_dtype out_dtype, int32_t accumulate,
                                       void* workspace, int64_t workspace_bytes, void* hip_stream)
{
    return gp::embedding_grad(tokens, index, N, grad, ldg, dtype, d, scale, V, table_grad, ldt, out_dtype, accumulate, workspace,
                              workspace_bytes, (hipStream_t)hip_stream);
}
