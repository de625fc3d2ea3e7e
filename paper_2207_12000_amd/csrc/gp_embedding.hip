// Embedding rows of a model over the hop stack, and their gradient.
//
//   lookup    out[i, :]  = scale * table[token[i], :]                      (zero where the token names no row)
//   gradient  grad[v, :] = scale * sum_{i: token[i] = v} up[i, :]
//
// The gradient is taken by sorted tokens: (token, position) pairs are sorted, which puts the positions of one token next to
// one another in ascending order, and the rows of up are summed along that list.  The list is cut into tiles of equal
// length whatever the tokens are, so a token that half of the positions name costs no more than any other; a token's
// run that a tile boundary cuts leaves one partial row in every tile it touches, and a second launch adds these up in
// tile order.  Every row of the gradient is written once: rows without a token get their zeros beside their neighbours.  Sums are held in
// fp32 and rounded once; what atomics there are count whole numbers, so the same inputs give the same bits.  Short lists take one launch
// instead, in which a workgroup has a range of the table's rows and all tokens that name them.
//
// What bounds it, and us measured.  Lookups of many rows: memory (2.45 M rows of 256 bf16 out of as many, 465 us, 1.25 GB written
// and as much asked for; 507,001 fp32 rows of 100 to bf16, 28 us); of few rows the launch (4,096 rows of 128, 4 us on the GPU).  Gradients of
// many rows: the gathered rows, each of which touches up to a 128-byte line more than it fills (2.45 M fp32 rows of 100 into as many,
// 563 - 590 us: sums 446 - 475, sort 106, joins and long gaps 17); of half a million the sort's four launches and the sums alike
// (bf16 rows of 100 into 32,768 rows by Zipf's law, 76 us: sort 37, sums 30, joins 9); of a few thousand one launch's chain of loads, places and
// sums, and the call (4,096 rows of 128 into 10,000, 12 us, 8.5 of them on the GPU; gp_sum_short).
#include <algorithm>
#include <exception>

#include "gp_internal.h"
#include "gp_rows.h"

namespace gp {

namespace {

constexpr int kThreads = 256;

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

// A launch takes fewer than 2^32 threads; workgroups beyond these walk on through the rest.
constexpr int64_t kMaxBlocks = 1 << 20;

template <typename TI, typename TO, int VEC>
gp_status launch_lookup(LookupArgs a, hipStream_t stream)
{
    a.nvec = (a.d + VEC - 1) / VEC;
    const int64_t blocks = (a.N * a.nvec + 4 * kThreads - 1) / (4 * kThreads);
    profile_begin("gp_embedding_rows", stream);
    hipLaunchKernelGGL((gp_embedding_rows<TI, TO, VEC>), dim3((unsigned)std::min(blocks, kMaxBlocks)), dim3(kThreads), 0, stream, a);
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

// The sort: least significant digit first, digits of up to 11 bits of the token, equal digits keep their order.  An entry is
// token << 32 | position; a token that names no row counts as V, behind all that do.  A pass of a long list: (1) every workgroup counts
// the digits of its tile of consecutive entries, (2) for every digit the tiles before each tile are added up, (3) every workgroup
// ranks its tile's entries -- a wavefront takes 64 at a time, finds the lanes with its own digit by one ballot per bit, and
// keeps counts of its own in LDS, so that no barrier stands between its steps -- and writes each to its place.
// (The sort that plans use, gp_device_sort.hip, is for long lists of keys that are there already: five launches a pass of 8 bits, tiles of 16,384
// keys, three barriers for every 256 of them.  507,001 tokens of 16 bits would take ten launches of up to 31 workgroups, and one to make the keys; here
// they take four launches, of 124.)
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kMaxDigits = 2048;

struct SortArgs {
    const void* tokens;    // the first pass reads these,
    int wide;
    const uint64_t* keys;  // the others these
    uint64_t* out;
    int64_t N, V;
    int shift, bits;       // the digit
    int64_t tiles;
    uint32_t* table;       // [tile][digit]
    uint32_t* totals;      // [digit]
    int own_table;         // no totals: the scatter adds up the table
};

__device__ __forceinline__ uint64_t entry_of(int64_t token, int64_t i, int64_t V)
{
    return (uint64_t)(token >= 0 && token < V ? token : V) << 32 | (uint64_t)i;
}
template <bool FIRST>
__device__ __forceinline__ uint64_t entry_at(const SortArgs& a, int64_t i)
{
    if constexpr (FIRST)
        return entry_of(token_at(a.tokens, a.wide, i), i, a.V);
    else
        return a.keys[i];
}

// lanes of the wavefront that are valid and hold the same digit
template <int BITS>
__device__ __forceinline__ unsigned long long peers_of(unsigned digit, bool valid)
{
    unsigned long long peers = __ballot(valid);
#pragma unroll
    for (int b = 0; b < BITS; ++b) {
        const bool bit = (digit >> b) & 1u;
        const unsigned long long with = __ballot(bit);
        peers &= bit ? with : ~with;
    }
    return peers;
}

// Ranks a wavefront's next 64 entries among its own; count: the wavefront's digit counts in LDS (volatile: its lanes hand them on
// without a barrier).
template <int BITS>
__device__ __forceinline__ uint32_t rank_in_wave(volatile uint16_t* count, unsigned digit, bool valid, int lane)
{
    const unsigned long long peers = peers_of<BITS>(digit, valid);
    const uint32_t before = (uint32_t)__popcll(peers & ((1ull << lane) - 1ull));
    uint32_t r = 0;
    if (valid) {
        r = count[digit] + before;
        if (before == 0) count[digit] = (uint16_t)(r + (uint32_t)__popcll(peers));
    }
    __builtin_amdgcn_wave_barrier();
    return r;
}

// exclusive prefix of v over the workgroup's threads; part: kSortWaves words of LDS
__device__ __forceinline__ uint32_t exclusive_1024(uint32_t v, uint32_t* part)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t incl = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t up = __shfl_up(incl, o, 64);
        if (lane >= o) incl += up;
    }
    __syncthreads();
    if (lane == 63) part[wave] = incl;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < wave; ++w) before += part[w];
    return before + incl - v;
}

template <int ITEMS, bool FIRST>
__global__ __launch_bounds__(kSortThreads) void gp_token_count(SortArgs a)
{
    __shared__ uint32_t h[kMaxDigits];
    const int digits = 1 << a.bits;
    const int64_t t0 = (int64_t)blockIdx.x * (ITEMS * kSortThreads) + threadIdx.x;
    unsigned digit[ITEMS];
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) digit[j] = t0 + j * kSortThreads < a.N ? (unsigned)(entry_at<FIRST>(a, t0 + j * kSortThreads) >> a.shift) & (digits - 1) : ~0u;
    for (int i = threadIdx.x; i < digits; i += kSortThreads) h[i] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
        if (digit[j] != ~0u) atomicAdd(&h[digit[j]], 1u);
    __syncthreads();
    for (int i = threadIdx.x; i < digits; i += kSortThreads) a.table[(int64_t)blockIdx.x * digits + i] = h[i];
}

// Where the table is small (kOwnTable entries), every scatter adds it up itself: 127 KB from an L2 (507,001 tokens of 16 bits) take it 4 us
// longer, a launch for it takes 5 and its place in the queue.
constexpr int64_t kOwnTable = 1 << 16;

// A workgroup looks after kPrefixDigits digits: its threads stand side by side over them, and each row of threads over a range of tiles.
constexpr int kPrefixDigits = 32, kPrefixRows = kSortThreads / kPrefixDigits;

__global__ __launch_bounds__(kSortThreads) void gp_token_prefix(SortArgs a)
{
    __shared__ uint32_t sums[kPrefixRows][kPrefixDigits];
    const int col = threadIdx.x % kPrefixDigits, row = threadIdx.x / kPrefixDigits;
    const int64_t digits = 1 << a.bits, d = (int64_t)blockIdx.x * kPrefixDigits + col;
    const int64_t each = (a.tiles + kPrefixRows - 1) / kPrefixRows, t0 = min(row * each, a.tiles), t1 = min(t0 + each, a.tiles);
    uint32_t sum = 0;
    if (d < digits)
#pragma unroll 8
        for (int64_t t = t0; t < t1; ++t) sum += a.table[t * digits + d];
    sums[row][col] = sum;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (int r = 0; r < kPrefixRows; ++r) {
        const uint32_t v = sums[r][col];
        before += r < row ? v : 0, all += v;
    }
    if (d >= digits) return;
    if (row == 0) a.totals[d] = all;
#pragma unroll 8
    for (int64_t t = t0; t < t1; ++t) {
        const uint32_t v = a.table[t * digits + d];
        a.table[t * digits + d] = before;
        before += v;
    }
}

// LDS of a scatter: what leads from an entry's place among the workgroup's to its place in the list, by digit; then counts [wave][digit],
// at first of the wavefront's own entries, later the place of its first one (a tile has fewer than 2^16); then, over these, the
// workgroup's entries in the new order: neighbours there are neighbours in the list, and their stores share lines.
constexpr size_t scatter_lds(int digits, int items)
{
    const size_t counts = (size_t)digits * 2 * kSortWaves, entries = (size_t)items * kSortThreads * 8;
    return kSortWaves * 4 + (size_t)digits * 4 + (counts > entries ? counts : entries);
}

template <int BITS, int ITEMS, bool FIRST>
__global__ __launch_bounds__(kSortThreads) void gp_token_scatter(SortArgs a)
{
    extern __shared__ __align__(16) uint32_t sort_lds[];
    constexpr int digits = 1 << BITS;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t *const part = sort_lds, *const lead = part + kSortWaves;
    uint16_t* const count = (uint16_t*)(lead + digits);
    uint64_t* const list = (uint64_t*)count;
    uint64_t key[ITEMS];
    uint32_t rank[ITEMS];
    const int64_t t0 = (int64_t)blockIdx.x * (ITEMS * kSortThreads), w0 = t0 + wave * (ITEMS * 64) + lane;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) key[j] = w0 + j * 64 < a.N ? entry_at<FIRST>(a, w0 + j * 64) : 0;
    // thread t looks after digits per t .. per t + per - 1: how many entries have them, and how many of those in the tiles before this one
    constexpr int per = (digits + kSortThreads - 1) / kSortThreads;
    const int d0 = threadIdx.x * per;
    uint32_t all[2] = {0, 0}, before[2] = {0, 0};
    static_assert(kMaxDigits == 2 * kSortThreads, "at most two digits per thread");
    if (per == 1 && a.own_table) {
        uint32_t(*const sums)[2] = (uint32_t(*)[2])list;
        const int d = threadIdx.x & (digits - 1), row = threadIdx.x / digits, rows = max(kSortThreads / digits, 1);
        uint32_t n = 0, b = 0;
#pragma unroll 8
        for (int t = row; t < (int)a.tiles; t += rows) {
            const uint32_t v = a.table[(int64_t)t * digits + d];
            n += v, b += t < (int)blockIdx.x ? v : 0;
        }
        sums[threadIdx.x][0] = n, sums[threadIdx.x][1] = b;
        __syncthreads();
        if (d0 < digits)
            for (int r = 0; r < rows; ++r) all[0] += sums[r * digits + d0][0], before[0] += sums[r * digits + d0][1];
        __syncthreads();
    } else {
#pragma unroll
        for (int j = 0; j < per; ++j)
            if (d0 + j < digits) all[j] = a.totals[d0 + j], before[j] = a.table[(int64_t)blockIdx.x * digits + d0 + j];
    }
    for (int i = threadIdx.x; i < kSortWaves / 2 * digits; i += kSortThreads) ((uint32_t*)count)[i] = 0;
    uint32_t begin = exclusive_1024(all[0] + all[1], part);
    if (d0 < digits) lead[d0] = begin + before[0];
    if (per > 1 && d0 + 1 < digits) lead[d0 + 1] = begin + all[0] + before[1];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
        rank[j] = rank_in_wave<BITS>(count + wave * digits, (unsigned)(key[j] >> a.shift) & (digits - 1), w0 + j * 64 < a.N, lane);
    __syncthreads();
    uint32_t mine = 0;
#pragma unroll
    for (int j = 0; j < per; ++j)
        if (d0 + j < digits)
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) mine += count[w * digits + d0 + j];
    begin = exclusive_1024(mine, part);
#pragma unroll
    for (int j = 0; j < per; ++j) {
        const int d = d0 + j;
        if (d >= digits) break;
        lead[d] -= begin;
        uint32_t n[kSortWaves];
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) n[w] = count[w * digits + d];
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) count[w * digits + d] = (uint16_t)begin, begin += n[w];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
        if (w0 + j * 64 < a.N) rank[j] += count[wave * digits + ((unsigned)(key[j] >> a.shift) & (digits - 1))];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
        if (w0 + j * 64 < a.N) list[rank[j]] = key[j];
    __syncthreads();
    const int here = (int)min((int64_t)ITEMS * kSortThreads, a.N - t0);
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
        const int i = j * kSortThreads + threadIdx.x;
        if (i >= here) continue;
        const uint64_t k = list[i];
        const uint32_t place = lead[(unsigned)(k >> a.shift) & (digits - 1)] + (uint32_t)i;
        if (place < a.N) a.out[place] = k;  // (always true)
    }
}

// A short list takes its places by counting, for every entry, those that are smaller (entries are all different): N^2 comparisons,
// but one launch (4,096 tokens 8 us; a radix sort by one workgroup took 14).  A workgroup ranks 64 entries, one per lane, against the whole
// list in LDS, a sixteenth of it per wavefront.
constexpr int64_t kShortList = 8192;

// how many of list[j0 .. j1) are below `own`, or, where EQUAL, not above it; j0, j1 multiples of 16
template <bool EQUAL>
__device__ __forceinline__ uint32_t count_below(const uint32_t* list, int j0, int j1, uint32_t own)
{
    uint32_t n = 0;
    for (int j = j0; j < j1; j += 16) {
        uint4 t[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) t[u] = *(const uint4*)(list + j + 4 * u);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            n += EQUAL ? (t[u].x <= own) + (t[u].y <= own) + (t[u].z <= own) + (t[u].w <= own) : (t[u].x < own) + (t[u].y < own) + (t[u].z < own) + (t[u].w < own);
    }
    return n;
}

__global__ __launch_bounds__(kSortThreads) void gp_token_rank(SortArgs a)
{
    __shared__ __align__(16) uint32_t list[kShortList];
    __shared__ uint32_t smaller[kSortWaves][64];
    const int N = (int)a.N, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int all = (N + 63) / 64 * 64;  // (behind the list: tokens above any)
    for (int i = threadIdx.x; i < all; i += kSortThreads) list[i] = i < N ? (uint32_t)(entry_at<true>(a, i) >> 32) : 0xFFFFFFFFu;
    __syncthreads();
    const int i0 = blockIdx.x * 64, i = i0 + lane;
    const int each = ((all + kSortWaves - 1) / kSortWaves + 15) / 16 * 16, j0 = min(wave * each, all), j1 = min(j0 + each, all);
    const uint32_t own = list[i];
    // before the workgroup's own entries an equal token is the smaller entry, behind them it is not
    uint32_t n = count_below<true>(list, j0, min(j1, i0), own) + count_below<false>(list, max(j0, i0 + 64), j1, own);
    if (wave == 0)
#pragma unroll 16
        for (int u = 0; u < 64; ++u) {
            const uint32_t t = __builtin_amdgcn_readlane(own, u);
            n += t < own || (t == own && u < lane);
        }
    smaller[wave][lane] = n;
    __syncthreads();
    if (wave > 0 || i >= N) return;
    uint32_t place = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) place += smaller[w][lane];
    if (place < (uint32_t)N) a.out[place] = (uint64_t)own << 32 | (uint64_t)i;  // (always true)
}

struct GradArgs {
    const uint64_t* keys;  // sorted
    int64_t N, V, tile, tiles;  // places of a tile (before the launch: of a stretch of it)
    const void* up;
    int64_t ldg;
    int d, nvec;
    float scale;
    void* out;
    int64_t ldt;
    int accumulate;
    float* carry;  // two partial rows of nvec vectors per tile: of the run that came in, of the run that goes on
    int64_t gap;   // rows (gap_rows)
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

// Rows of zeros: those of a gap in the tokens that is at most `gap` rows long are written beside the run behind it, others by gp_join_tiles.
// A lane that writes a gap does so row after row, so that long ones are left to the others where there are many (gaps of up to 256 and up to
// 32 rows, us: 5 k tokens in 200 k rows of 64 36 / 28, 10 k in 1 M rows of 100 131 / 117, 100 k in 2.4 M rows of 64 186 / 172); where the mean
// gap is shorter than 16 rows, looking for them costs as much or more (100 k in 1.7 M 146 / 147, in 1 M 98 / 109).
int64_t gap_rows(int64_t N, int64_t V) { return V > 16 * N ? 32 : 256; }

// G lanes walk one stretch of a.tile / kGroups places, a lane holds one vector of the sums; the workgroup's stretches are one tile.  A run
// that goes on from stretch to stretch is put together by the lanes in whose stretch it begins (or, where it came into the tile, by
// the first ones), from what the others leave in LDS; only what leaves the tile goes through memory.
template <typename TG, typename TO, int VEC, int G, int THREADS>
__device__ __forceinline__ void sum_tile(const GradArgs& a, const uint64_t* keys, int64_t tile, float (*head)[VEC], int* passes)
{
    constexpr int U = 8, kGroups = THREADS / G;
    const int g = threadIdx.x / G, c = blockIdx.y * G + threadIdx.x % G;
    const int64_t stretch = a.tile / kGroups, lo = tile * a.tile + g * stretch, hi = min(lo + stretch, a.N);
    const bool active = c < a.nvec;
    const int col = min(min(c, a.nvec - 1) * VEC, a.d - VEC);
    const TG* const up = (const TG*)a.up + col;
    float* const carry = a.carry + (2 * tile * a.nvec + c) * VEC;  // of the run that came in; the other's is one row on
    float acc[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = 0.0f;
    auto fill_gap = [&](int64_t before, int64_t token) {
        if (a.accumulate || token >= a.V || token - before > a.gap + 1) return;
        float zero[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) zero[i] = 0.0f;
        for (int64_t r = before + 1; r < token; ++r) store_vec<TO, VEC>((TO*)a.out + r * a.ldt + col, zero);
    };
    int64_t cur = a.V;
    bool came_in = false, open = false;
    if (lo < a.N && active) {
        cur = (int64_t)(keys[lo] >> 32);
        if (lo > 0) {
            const int64_t before = (int64_t)(keys[lo - 1] >> 32);
            came_in = before == cur;
            if (!came_in) fill_gap(before, cur);
        }
        uint64_t key[U];
#pragma unroll
        for (int u = 0; u < U; ++u) key[u] = lo + u < hi ? keys[lo + u] : ~UINT64_C(0);
        for (int64_t p = lo; p < hi; p += U) {
            typename Vec<TG, VEC>::type v[U];  // (widened when they are added: registers decide how many wavefronts there are)
            uint64_t next[U];                  // (asked for beside this step's rows, not behind them)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                v[u] = 0;
                if ((int64_t)(key[u] >> 32) < a.V) v[u] = *reinterpret_cast<const typename Vec<TG, VEC>::type*>(up + (int64_t)(key[u] & 0xFFFFFFFFu) * a.ldg);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) next[u] = p + U + u < hi ? keys[p + U + u] : ~UINT64_C(0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (p + u >= hi) break;
                const int64_t tok = (int64_t)(key[u] >> 32);
                if (tok != cur) {  // (cur < tok <= V)
                    if (!came_in)
                        finish<TO, VEC>(a, cur, c, acc);
                    else if (g == 0)
                        store_vec<float, VEC>(carry, acc);
                    else
                        store_vec<float, VEC>(head[threadIdx.x], acc);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) acc[i] = 0.0f;
                    fill_gap(cur, tok);
                    cur = tok, came_in = false;
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[i] += element<TG, VEC>(v[u], i);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) key[u] = next[u];
        }
        open = cur < a.V && hi < a.N && (int64_t)(keys[hi] >> 32) == cur;
        if (came_in && g > 0) {
            store_vec<float, VEC>(head[threadIdx.x], acc);
            if (threadIdx.x % G == 0) passes[g] = open;
            cur = a.V;  // (another's run)
        } else if (threadIdx.x % G == 0) {
            passes[g] = false;
        }
    }
    __syncthreads();
    if (cur >= a.V) return;
    if (open)
        for (int h = g + 1; h < kGroups && open; ++h) {
            float v[VEC];
            load_vec<float, VEC>(head[h * G + threadIdx.x % G], v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) acc[i] += v[i];
            open = passes[h];
        }
    if (came_in)
        store_vec<float, VEC>(carry, acc);
    else if (open)
        store_vec<float, VEC>(carry + (int64_t)a.nvec * VEC, acc);
    else
        finish<TO, VEC>(a, cur, c, acc);
}

template <typename TG, typename TO, int VEC, int G>
__global__ __launch_bounds__(kThreads) void gp_sum_tiles(GradArgs a)
{
    __shared__ float head[kThreads][VEC];    // what a stretch adds to the run that comes into it
    __shared__ int passes[kThreads / G];     // that run goes on behind the stretch
    sum_tile<TG, TO, VEC, G, kThreads>(a, a.keys, blockIdx.x, head, passes);
}

// the first place of the sorted list whose token is not below v, by all lanes of a wavefront (64 probes a round)
__device__ __forceinline__ int64_t first_not_below(const uint64_t* keys, int64_t N, int64_t v, int lane)
{
    int64_t lo = 0, n = N;  // it lies in lo .. lo + n
    while (n > 0) {
        const int64_t step = (n + 64) / 65, p = lo + (lane + 1) * step - 1;
        const int below = __popcll(__ballot(p < lo + n && (int64_t)(keys[p < lo + n ? p : lo] >> 32) < v));
        lo += below * step, n = below == 64 ? n - 64 * step : min(step - 1, n - below * step);
    }
    return lo;
}

// zeros in rows [r, end), by the lanes of a wavefront
template <typename TO>
__device__ __forceinline__ void zero_rows(const GradArgs& a, int64_t r, int64_t end, int lane)
{
    constexpr int N = 16 / sizeof(TO);
    float zero[N];
#pragma unroll
    for (int i = 0; i < N; ++i) zero[i] = 0.0f;
    const bool whole = a.ldt == a.d;  // one stretch
    const int64_t len = whole ? max((end - r) * a.d, (int64_t)0) : a.d;
    for (; r < end; r = whole ? end : r + 1) {
        TO* const p = (TO*)a.out + r * a.ldt;
        for (int64_t i = (int64_t)lane * N; i + N <= len; i += 64 * N) store_vec<TO, N>(p + i, zero);
        const int64_t i = len - len % N + lane;
        if (i < len) p[i] = 0;
    }
}

template <typename TO>
__global__ __launch_bounds__(kThreads) void gp_zero_table(GradArgs a)
{
    constexpr int kWaves = kThreads / 64;
    const int64_t per = (a.V + gridDim.x * kWaves - 1) / (gridDim.x * kWaves), r0 = ((int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6)) * per;
    zero_rows<TO>(a, min(r0, a.V), min(r0 + per, a.V), threadIdx.x & 63);
}

// Short lists in one launch: a workgroup has a range of the table's rows.  It reads all tokens, keeps those of its rows in LDS in their order,
// sorts them there by row, writes zeros to its rows without a token and sums up the others as one tile.
// Three dependent launches (places by counting, sums, joins) take longer the shorter the list is: us on the GPU, three launches / one,
// 500 x 64 into 300 rows 10.8 / 5.9, 4096 x 128 into 1000 16.3 / 7.4, the same by Zipf's law 17.7 / 16.3, into 60 rows 16.7 / 9.6, into
// 100 k 24.5 / 13.6.  But a token's rows are one workgroup's: 4096 x 128 of one token take 18 / 29 with 32 rows, 18 / 33 with 1000, 19 / 42 with 10,000, so
// lists of more than 128 tokens per row of the table, or of more than a million elements (4096 x 602: 17 / 17, of one token 36 / 84), go the
// other way.  4,096 tokens are what one count per lane of a wavefront holds (divide below), no limit of the method: 4,097 take 17.5, 8,192 22.4.
constexpr int kShortThreads = 1024, kShortBlocks = 256;
constexpr int64_t kShortest = 4096, kShortElements = 1 << 20, kShortPerRow = 128;
constexpr int kCounted = 128;  // tokens of a workgroup up to which each one's place is counted; beyond, they are sorted bit by bit of the row

template <typename TG, typename TO, int VEC, int G>
__global__ __launch_bounds__(kShortThreads) void gp_sum_short(GradArgs a, const void* tokens, int wide)
{
    constexpr int kGroups = kShortThreads / G, kLoads = kShortest / kShortThreads, kWaves = kShortThreads / 64;
    static_assert(kLoads * kWaves <= 64, "a lane has one count");
    extern __shared__ __align__(16) char lds[];
    __shared__ int passes[kGroups];
    __shared__ int counts[2][kLoads * kWaves];
    float(*const head)[VEC] = (float(*)[VEC])lds;
    uint64_t* const keys = (uint64_t*)(lds + sizeof(float) * VEC * kShortThreads);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t r0 = a.V * blockIdx.x / gridDim.x, r1 = a.V * (blockIdx.x + 1) / gridDim.x;
    int64_t token[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        const int64_t i = threadIdx.x + k * kShortThreads;
        token[k] = i >= a.N ? -1 : wide ? ((const int64_t*)tokens)[i] : (int64_t)((const int32_t*)tokens)[i];
    }
    // `members` of the items (one per thread and k, their order) to the front, the others behind them, both in order; returns how many
    auto divide = [&](const bool (&member)[kLoads], const bool (&other)[kLoads], const uint64_t (&item)[kLoads], int loads) {
        uint64_t in[kLoads], out[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k)
            if (k < loads) {
                in[k] = __ballot(member[k]), out[k] = __ballot(other[k]);
                if (lane == 0) counts[0][k * kWaves + wave] = __popcll(in[k]), counts[1][k * kWaves + wave] = __popcll(out[k]);
            }
        __syncthreads();  // (and every item has been read)
        const int slots = loads * kWaves;
        int x = lane < slots ? counts[0][lane] : 0, y = lane < slots ? counts[1][lane] : 0;
#pragma unroll
        for (int step = 1; step < 64; step *= 2) {
            const int xs = __shfl_up(x, step), ys = __shfl_up(y, step);
            if (lane >= step) x += xs, y += ys;
        }
        const int members = __shfl(x, 63);
        const uint64_t below = (UINT64_C(1) << lane) - 1;
#pragma unroll
        for (int k = 0; k < kLoads; ++k)
            if (k < loads) {
                const int slot = k * kWaves + wave;
                const int x0 = __shfl(x, slot) - __popcll(in[k]), y0 = members + __shfl(y, slot) - __popcll(out[k]);
                if (member[k]) keys[x0 + __popcll(in[k] & below)] = item[k];
                if (other[k]) keys[y0 + __popcll(out[k] & below)] = item[k];
            }
        __syncthreads();
        return members;
    };
    bool member[kLoads], other[kLoads];
    uint64_t item[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        member[k] = token[k] >= r0 && token[k] < r1, other[k] = false;
        item[k] = (uint64_t)token[k] << 32 | (uint64_t)(threadIdx.x + k * kShortThreads);
    }
    const int count = divide(member, other, item, (int)((a.N + kShortThreads - 1) / kShortThreads));
    if (count <= kCounted) {  // an item's place: how many are smaller
        int place = 0;
        const uint64_t x = threadIdx.x < count ? keys[threadIdx.x] : 0;
        if (threadIdx.x < count)
            for (int i = 0; i < count; ++i) place += keys[i] < x;
        __syncthreads();
        if (threadIdx.x < count) keys[place] = x;
        __syncthreads();
    } else {  // bit by bit of the row
        for (int bit = 0; (r1 - r0 - 1) >> bit; ++bit) {
#pragma unroll
            for (int k = 0; k < kLoads; ++k) {
                const int i = threadIdx.x + k * kShortThreads;
                const bool here = i < count;
                item[k] = here ? keys[i] : 0;
                const bool one = (((int64_t)(item[k] >> 32) - r0) >> bit) & 1;
                member[k] = here && !one, other[k] = here && one;
            }
            divide(member, other, item, (count + kShortThreads - 1) / kShortThreads);
        }
    }
    const int share = (int)min((r1 - r0 + kWaves - 1) / kWaves, (int64_t)64);  // rows that a wavefront looks after at a time
    if (!a.accumulate && blockIdx.y == 0)
        for (int64_t r = r0 + wave * share; r < r1; r += kWaves * share) {
            int at = 0, n = count;  // the first place whose token is not below this lane's row
            while (n > 0) {
                const int half = n / 2;
                const bool below = (int64_t)(keys[at + half] >> 32) < r + lane;
                at = below ? at + half + 1 : at, n = below ? n - half - 1 : half;
            }
            uint64_t empty = __ballot(lane < share && r + lane < r1 && !(at < count && (int64_t)(keys[at] >> 32) == r + lane));
            while (empty) {
                const int first = __builtin_ctzll(empty);
                const uint64_t rest = ~(empty >> first);
                const int rows = rest ? __builtin_ctzll(rest) : 64;  // (all 64: nothing is shifted in)
                zero_rows<TO>(a, r + first, r + first + rows, lane);
                empty = first + rows >= 64 ? 0 : empty >> (first + rows) << (first + rows);
            }
        }
    if (count == 0) return;
    GradArgs mine = a;  // (no gap is left to be filled beside a run)
    mine.N = count, mine.tile = (count + kGroups - 1) / kGroups * kGroups, mine.gap = 0;
    sum_tile<TG, TO, VEC, G, kShortThreads>(mine, keys, 0, head, passes);
}

// Wavefronts behind the tiles' workgroups look after a.gap rows each and walk on through the table: a gap of more rows than that, or one before the first token or behind
// the last, covers at most the rows up to the first token among them and those behind the last.
template <typename TO>
__device__ __forceinline__ void fill_long_gaps(const GradArgs& a, int64_t chunk, int lane)
{
    const int64_t r0 = chunk * a.gap, r1 = min(r0 + a.gap, a.V);
    const int64_t p = first_not_below(a.keys, a.N, r0, lane), q = first_not_below(a.keys, a.N, r1, lane);
    const int64_t before = p > 0 ? (int64_t)(a.keys[p - 1] >> 32) : -1, first = p < a.N ? min((int64_t)(a.keys[p] >> 32), a.V) : a.V;
    if (p == 0 || first == a.V || first - before > a.gap + 1) zero_rows<TO>(a, r0, min(first, r1), lane);
    if (first >= r1) return;
    const int64_t last = (int64_t)(a.keys[q - 1] >> 32), next = q < a.N ? min((int64_t)(a.keys[q] >> 32), a.V) : a.V;
    if (next == a.V || next - last > a.gap + 1) zero_rows<TO>(a, last + 1, r1, lane);
}

// Runs that go on into other tiles.  G lanes look at one tile: where such a run begins in it, its partial rows are added up in tile order;
// a run of more than kShortRun further tiles is left to the whole workgroup, whose groups take every kGroups-th tile each.
constexpr int kShortRun = 8;

template <typename TO, int VEC, int G>
__global__ __launch_bounds__(kThreads) void gp_join_tiles(GradArgs a, int64_t tile_blocks)
{
    constexpr int kGroups = kThreads / G;
    __shared__ float part[kThreads][VEC];
    __shared__ int64_t longer[kGroups];
    __shared__ int longer_count;
    if (blockIdx.x >= tile_blocks) {
        constexpr int kWaves = kThreads / 64;
        if (blockIdx.y > 0) return;
        for (int64_t chunk = (blockIdx.x - tile_blocks) * kWaves + (threadIdx.x >> 6); chunk * a.gap < a.V; chunk += (gridDim.x - tile_blocks) * kWaves)
            fill_long_gaps<TO>(a, chunk, threadIdx.x & 63);
        return;
    }
    if (threadIdx.x == 0) longer_count = 0;
    __syncthreads();
    const int g = threadIdx.x / G, c = blockIdx.y * G + threadIdx.x % G;
    const int64_t row = (int64_t)a.nvec * VEC, at = (int64_t)c * VEC;  // floats of a partial row; this lane's place in it
    const int64_t t = (int64_t)blockIdx.x * kGroups + g, lo = t * a.tile, hi = lo + a.tile;
    if (hi < a.N) {
        const int64_t tok = (int64_t)(a.keys[hi - 1] >> 32);
        const bool begins = lo == 0 || (int64_t)(a.keys[lo - 1] >> 32) != tok;
        if (tok < a.V && begins && (int64_t)(a.keys[hi] >> 32) == tok) {
            int more = 0;  // tiles that start with the token
#pragma unroll
            for (int i = 0; i <= kShortRun; ++i) {
                const int64_t p = hi + i * a.tile;
                more += p < a.N && (int64_t)(a.keys[p] >> 32) == tok;
            }
            if (more > kShortRun) {
                if (threadIdx.x % G == 0) longer[atomicAdd(&longer_count, 1)] = t;
            } else if (c < a.nvec) {
                float acc[VEC], v[kShortRun][VEC];
                load_vec<float, VEC>(a.carry + (2 * t + 1) * row + at, acc);
#pragma unroll
                for (int i = 0; i < kShortRun; ++i) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) v[i][e] = 0.0f;
                    if (i < more) load_vec<float, VEC>(a.carry + 2 * (t + 1 + i) * row + at, v[i]);
                }
#pragma unroll
                for (int i = 0; i < kShortRun; ++i)
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if (i < more) acc[e] += v[i][e];
                finish<TO, VEC>(a, tok, c, acc);
            }
        }
    }
    __syncthreads();
    const int count = longer_count;
    for (int k = 0; k < count; ++k) {
        const int64_t t = longer[k];
        const int64_t tok = (int64_t)(a.keys[t * a.tile + a.tile - 1] >> 32);
        int64_t first = t + 1, last = a.tiles;  // the first tile whose list does not start with the token: between these
        while (first < last) {
            const int64_t mid = (first + last) / 2;
            if ((int64_t)(a.keys[mid * a.tile] >> 32) == tok) first = mid + 1;
            else last = mid;
        }
        float acc[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] = 0.0f;
        if (c < a.nvec) {
            if (g == 0) load_vec<float, VEC>(a.carry + (2 * t + 1) * row + at, acc);
            constexpr int U = 8;
            for (int64_t s = t + 1 + g; s < last; s += U * kGroups) {
                float v[U][VEC];
#pragma unroll
                for (int u = 0; u < U; ++u) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) v[u][e] = 0.0f;
                    if (s + u * kGroups < last) load_vec<float, VEC>(a.carry + 2 * (s + u * kGroups) * row + at, v[u]);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) acc[e] += v[u][e];
            }
        }
        __syncthreads();  // (the run before is read to its end)
#pragma unroll
        for (int e = 0; e < VEC; ++e) part[threadIdx.x][e] = acc[e];
        __syncthreads();
        if (g > 0 || c >= a.nvec) continue;
        for (int o = 1; o < kGroups; ++o)
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[e] += part[o * G + threadIdx.x][e];
        finish<TO, VEC>(a, tok, c, acc);
    }
}

template <typename TG, typename TO, int VEC, int G>
gp_status launch_sums(GradArgs a, const void* tokens, int wide, hipStream_t stream)
{
    const unsigned ny = (unsigned)((a.nvec + G - 1) / G);
    if (tokens) {
        const size_t lds = sizeof(float) * VEC * kShortThreads + 8 * (size_t)a.N;
        gp_status st = raise_lds<&gp_sum_short<TG, TO, VEC, G>>(sizeof(float) * VEC * kShortThreads + 8 * kShortest);
        if (st != GP_OK) return st;
        profile_begin("gp_sum_short", stream);
        hipLaunchKernelGGL((gp_sum_short<TG, TO, VEC, G>), dim3((unsigned)std::min<int64_t>(a.V, kShortBlocks), ny), dim3(kShortThreads), lds, stream, a, tokens, wide);
        profile_end(stream);
        GP_HIP(hipGetLastError());
        return GP_OK;
    }
    constexpr int per = kThreads / G;
    a.tile *= per, a.tiles = (a.N + a.tile - 1) / a.tile;
    profile_begin("gp_sum_tiles", stream);
    hipLaunchKernelGGL((gp_sum_tiles<TG, TO, VEC, G>), dim3((unsigned)a.tiles, ny), dim3(kThreads), 0, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    const int64_t fills = a.accumulate ? 0 : std::min(((a.V + a.gap - 1) / a.gap + kThreads / 64 - 1) / (kThreads / 64), kMaxBlocks);
    if (a.tiles > 1 || fills > 0) {
        profile_begin("gp_join_tiles", stream);
        const int64_t tile_blocks = (a.tiles + per - 1) / per;
        hipLaunchKernelGGL((gp_join_tiles<TO, VEC, G>), dim3((unsigned)(tile_blocks + fills), ny), dim3(kThreads), 0, stream, a, tile_blocks);
        profile_end(stream);
        GP_HIP(hipGetLastError());
    }
    return GP_OK;
}
template <typename TG, typename TO, int VEC>
gp_status launch_sums(GradArgs a, const void* tokens, int wide, hipStream_t stream)
{
    a.nvec = (a.d + VEC - 1) / VEC;
    if (a.nvec <= 8) return launch_sums<TG, TO, VEC, 8>(a, tokens, wide, stream);
    if (a.nvec <= 16) return launch_sums<TG, TO, VEC, 16>(a, tokens, wide, stream);
    if (a.nvec <= 32) return launch_sums<TG, TO, VEC, 32>(a, tokens, wide, stream);
    return launch_sums<TG, TO, VEC, 64>(a, tokens, wide, stream);
}
template <typename TG, typename TO>
gp_status launch_sums(const GradArgs& a, const void* tokens, int wide, hipStream_t stream)
{
    constexpr int VEC = sizeof(TG) == 2 ? 8 : 4;
    return a.d >= VEC ? launch_sums<TG, TO, VEC>(a, tokens, wide, stream) : launch_sums<TG, TO, 1>(a, tokens, wide, stream);
}

// Stretches: equal lengths; enough of them to fill the chip, few enough that the partial rows of one token are added up fast.
// (2.45 M rows of 100: 563 us with 16,384, 588 with 32,768, 591 with 8,192.)
constexpr int64_t kMinStretch = 4, kMaxStretches = 16384;
int64_t stretch_length(int64_t N) { return std::max(kMinStretch, (N + kMaxStretches - 1) / kMaxStretches); }

int bits_of(int64_t v)
{
    int b = 0;
    while (v >> b) ++b;
    return b;
}

// the digits of tokens 0 .. V (V: those that name no row)
struct SortPlan {
    int passes, bits, items;
    int64_t tiles;
};
SortPlan sort_plan(int64_t N, int64_t V)
{
    SortPlan p;
    const int all = bits_of(V);
    p.passes = (all + 10) / 11;
    const int least = (all + p.passes - 1) / p.passes;
    p.bits = least <= 6 ? 6 : least <= 8 ? 8 : least == 9 ? 9 : 11;  // (those that the scatter is built for)
    p.items = N <= (1 << 20) ? 4 : 16;
    p.tiles = (N + p.items * kSortThreads - 1) / (p.items * kSortThreads);
    return p;
}

struct GradLayout {
    int64_t other, table, totals, carry, total;
};
GradLayout grad_layout(int64_t N, int64_t V, int32_t d)
{
    auto up = [](int64_t b) { return (b + 255) / 256 * 256; };
    const int64_t tile = stretch_length(N) * 4, tiles = (N + tile - 1) / tile;  // (four stretches to a tile, or more)
    const SortPlan p = sort_plan(N, V);
    GradLayout l;
    l.other = up(8 * N);
    l.table = l.other + up(N <= kShortList ? 0 : 8 * N);
    l.totals = l.table + up(N <= kShortList ? 0 : (p.tiles << p.bits) * 4);
    l.carry = l.totals + up(N <= kShortList ? 0 : (4 << p.bits));
    l.total = l.carry + up(2 * tiles * (((int64_t)d + 7) / 8 * 8) * 4);
    return l;
}

template <int BITS, int ITEMS, bool FIRST>
gp_status launch_scatter(const SortArgs& a, hipStream_t stream)
{
    constexpr size_t lds = scatter_lds(1 << BITS, ITEMS);
    gp_status st = raise_lds<&gp_token_scatter<BITS, ITEMS, FIRST>>(lds);
    if (st != GP_OK) return st;
    profile_begin("gp_token_scatter", stream);
    hipLaunchKernelGGL((gp_token_scatter<BITS, ITEMS, FIRST>), dim3((unsigned)a.tiles), dim3(kSortThreads), lds, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    return GP_OK;
}
template <int ITEMS, bool FIRST>
gp_status launch_pass(const SortArgs& a, hipStream_t stream)
{
    profile_begin("gp_token_count", stream);
    hipLaunchKernelGGL((gp_token_count<ITEMS, FIRST>), dim3((unsigned)a.tiles), dim3(kSortThreads), 0, stream, a);
    profile_end(stream);
    if (!a.own_table) {
        profile_begin("gp_token_prefix", stream);
        hipLaunchKernelGGL(gp_token_prefix, dim3((unsigned)(((1 << a.bits) + kPrefixDigits - 1) / kPrefixDigits)), dim3(kSortThreads), 0, stream, a);
        profile_end(stream);
    }
    GP_HIP(hipGetLastError());
    switch (a.bits) {
    case 6: return launch_scatter<6, ITEMS, FIRST>(a, stream);
    case 8: return launch_scatter<8, ITEMS, FIRST>(a, stream);
    case 9: return launch_scatter<9, ITEMS, FIRST>(a, stream);
    default: return launch_scatter<11, ITEMS, FIRST>(a, stream);
    }
}

// *sorted: whichever of the two lists of the workspace holds the result
gp_status sort_tokens(const void* tokens, int wide, int64_t N, int64_t V, char* ws, const GradLayout& l, hipStream_t stream, const uint64_t** sorted)
{
    const SortPlan p = sort_plan(N, V);
    SortArgs a{};
    a.tokens = tokens, a.wide = wide, a.N = N, a.V = V, a.bits = p.bits, a.tiles = p.tiles;
    a.table = (uint32_t*)(ws + l.table), a.totals = (uint32_t*)(ws + l.totals);
    a.own_table = p.bits <= 10 && p.tiles << p.bits <= kOwnTable;
    if (N <= kShortList) {
        a.out = (uint64_t*)ws;
        profile_begin("gp_token_rank", stream);
        hipLaunchKernelGGL(gp_token_rank, dim3((unsigned)((N + 63) / 64)), dim3(kSortThreads), 0, stream, a);
        profile_end(stream);
        GP_HIP(hipGetLastError());
        *sorted = a.out;
        return GP_OK;
    }
    uint64_t* lists[2] = {(uint64_t*)ws, (uint64_t*)(ws + l.other)};
    for (int pass = 0; pass < p.passes; ++pass) {
        a.shift = 32 + pass * p.bits, a.keys = lists[(pass + 1) & 1], a.out = lists[pass & 1];
        gp_status st = p.items == 4 ? (pass == 0 ? launch_pass<4, true>(a, stream) : launch_pass<4, false>(a, stream))
                                    : (pass == 0 ? launch_pass<16, true>(a, stream) : launch_pass<16, false>(a, stream));
        if (st != GP_OK) return st;
    }
    *sorted = a.out;
    return GP_OK;
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
    if (N < 0 || V < 1 || d < 1 || (ldg < d && ldg != 0) || ldt < d)
        return fail(GP_ERR_INVALID_ARG, "need N >= 0, V >= 1, d >= 1, ldg >= d or 0, ldt >= d");
    if (N > kMaxCount || V > kMaxCount) return fail(GP_ERR_UNSUPPORTED, "more than 2^31 - 1 tokens or rows");
    if (!out || (N > 0 && (!tokens || !up))) return fail(GP_ERR_INVALID_ARG, "NULL argument");
    const GradLayout l = grad_layout(N, V, d);
    if (N > 0 && (!workspace || bytes < l.total || (uintptr_t)workspace % 256 != 0))
        return fail(GP_ERR_INVALID_ARG, "need a workspace of %lld bytes on a 256-byte boundary", (long long)l.total);
    if (N == 0) {
        if (accumulate) return GP_OK;
        const unsigned grid = (unsigned)std::min<int64_t>((V + 3) / 4, 256 * 16);
        GradArgs a{};
        a.V = V, a.d = d, a.out = out, a.ldt = ldt;
        profile_begin("gp_zero_table", stream);
        if (out_dtype == GP_F32)
            hipLaunchKernelGGL(gp_zero_table<float>, dim3(grid), dim3(kThreads), 0, stream, a);
        else
            hipLaunchKernelGGL(gp_zero_table<bf16_t>, dim3(grid), dim3(kThreads), 0, stream, a);
        profile_end(stream);
        GP_HIP(hipGetLastError());
        return GP_OK;
    }
    char* const ws = (char*)workspace;
    GradArgs a{};
    a.N = N, a.V = V, a.tile = stretch_length(N), a.up = up, a.ldg = ldg, a.d = d, a.scale = scale, a.out = out, a.ldt = ldt,
    a.accumulate = accumulate != 0, a.carry = (float*)(ws + l.carry), a.gap = gap_rows(N, V);
    const int wide = index == GP_I64;
    const bool in_one = N <= kShortest && N * d <= kShortElements && N <= kShortPerRow * V;
    if (!in_one) {
        gp_status st = sort_tokens(tokens, wide, N, V, ws, l, stream, &a.keys);
        if (st != GP_OK) return st;
    }
    const void* const unsorted = in_one ? tokens : nullptr;
    if (dtype == GP_F32) return out_dtype == GP_F32 ? launch_sums<float, float>(a, unsorted, wide, stream) : launch_sums<float, bf16_t>(a, unsorted, wide, stream);
    return out_dtype == GP_F32 ? launch_sums<bf16_t, float>(a, unsorted, wide, stream) : launch_sums<bf16_t, bf16_t>(a, unsorted, wide, stream);
}

}  // namespace

}  // namespace gp

extern "C" gp_status gp_embedding(const void* table, int64_t ldt, gp_dtype dtype, int64_t V, int32_t d, const void* tokens, gp_index index,
                                  int64_t N, float scale, void* out, int64_t ldo, gp_dtype out_dtype, void* hip_stream)
{
    try {
        return gp::embedding(table, ldt, dtype, V, d, tokens, index, N, scale, out, ldo, out_dtype, (hipStream_t)hip_stream);
    } catch (const std::exception& e) {
        return gp::fail(GP_ERR_OOM_HOST, "gp_embedding: %s", e.what());
    }
}

extern "C" int64_t gp_embedding_grad_workspace(int64_t N, int64_t V, int32_t d)
{
    if (N < 0 || N > gp::kMaxCount || V < 1 || V > gp::kMaxCount || d < 1) return -1;
    return N == 0 ? 0 : gp::grad_layout(N, V, d).total;
}

extern "C" gp_status gp_embedding_grad(const void* tokens, gp_index index, int64_t N, const void* grad, int64_t ldg, gp_dtype dtype, int32_t d,
                                       float scale, int64_t V, void* table_grad, int64_t ldt, gp_dtype out_dtype, int32_t accumulate,
                                       void* workspace, int64_t workspace_bytes, void* hip_stream)
{
    try {
        return gp::embedding_grad(tokens, index, N, grad, ldg, dtype, d, scale, V, table_grad, ldt, out_dtype, accumulate, workspace,
                                  workspace_bytes, (hipStream_t)hip_stream);
    } catch (const std::exception& e) {
        return gp::fail(GP_ERR_OOM_HOST, "gp_embedding_grad: %s", e.what());
    }
}
