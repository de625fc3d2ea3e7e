// What rows of logits say, and what they learn from: log probabilities with entropies and alternatives, and a teacher's best logits, with their gradients.
//
//   answers   z = s x,  log p_j = z_j - log(sum exp z),  entropy = -sum p log p,  the k largest x
//   gradient  dx_j = s (g1 ([j = token] - p_j) - g2 p_j (log p_j + entropy))
//   distill   q = softmax(v / T) over a teacher's entries,  loss = T^2 sum q (log q - log p),  dx_j = g T (p_j - sum of q over entries that name j)
//
// With m the row's largest logit everything is a function of (x_j - m): sums are of exp(s (x_j - m)), which are at most 1, and log p_j is
// s (x_j - m) - log(sum), so that large logits cost no bits.  (m, log(sum)) are what a row's gradient needs.  A row whose logits are all -inf
// keeps (0, 0): every p is 0 and every log p is -inf, without a case of its own.
//
// All are bound by memory: a row is read once, into the registers of a team of lanes (as it is stored: widened it would take twice as many in bf16), and
// where the gradient is asked for along with the loss it is written from there.  Rows that a workgroup cannot hold, and few long rows, are cut into
// parts, a workgroup each, whose results a second launch joins.  us measured, and what the same bytes take a large copy: 4,096 rows of 32,768 in
// bf16, eight alternatives 63 (58), loss and gradient 109 (116); 507,001 fp32 rows of 47, loss and gradient 59 (49); the gradient of 2.45 M of them 200 (213).
//
// Alternatives.  Teams of part of a wavefront sort their elements in registers, put their lists together and keep the largest.  A logit and its class make
// one number there, larger logits and then lower classes first, so no two are equal (double_of, and key_of in memory).  Teams of a wavefront or more
// compare with a bound instead: the k-th largest of 64 groups' maxima is no larger than the k-th largest logit, and few others
// reach it (8.5 for 8, 44 for 32, in any order that does not follow the groups; of 256 groups 74 for 64); these are listed in LDS and ranked by counting.
// Where more reach it than the list has room for, as in rows of equal logits, the largest key below the last is looked for k times.
#include <algorithm>
#include <exception>

#include "gp_internal.h"
#include "gp_rows.h"

namespace gp {

namespace {

constexpr int kMostTop = 64;      // alternatives, and entries of a teacher: one to a lane of a wavefront
constexpr int kIndexBits = 28;    // of a class in a key
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr int kFewTop = 32;       // alternatives up to which 64 groups bound them: 8.5 logits reach the bound for 8, 44 for 32
constexpr int kRoom = 1024;       // keys that a workgroup's list has room for (a wavefront's: a quarter)

struct AnswerArgs {
    const void* x;
    int64_t ld, N;
    int C, nvec;
    const void* tokens;
    int wide;
    float scale;
    float *logp, *entropy, *stats;
    int k;
    int32_t* top_index;
    float* top_logp;
    int parts;      // of a row; more than one: results go to `partial`
    float* partial;  // [N][parts][4]: largest, sum of exp, sum of z exp; then [N][parts][k] keys
    uint64_t* keys;
};

__device__ __forceinline__ float infinity() { return __builtin_inff(); }

// max of floats that are no NaN's business: what is larger by the instruction (NaN is passed over)
__device__ __forceinline__ float larger(float a, float b)
{
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
template <int W>
__device__ __forceinline__ float team_largest(float v)
{
    return team<W>(v, [](float a, float b) { return larger(a, b); });
}

// Larger logits first (NaN above infinity, 0 and -0 the same), lower classes among equals.  60 bits: as a double a positive number, whose order is theirs.
__device__ __forceinline__ uint64_t key_of(float x, int j)
{
    const unsigned b = __float_as_uint(x + 0.0f);
    const unsigned o = x != x ? 0xFFFFFFFFu : b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
    return ((uint64_t)o << kIndexBits) | (uint64_t)((1u << kIndexBits) - 1 - j);
}
__device__ __forceinline__ float logit_of(uint64_t key)
{
    const unsigned o = (unsigned)(key >> kIndexBits);
    return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);  // (NaN gives NaN)
}
__device__ __forceinline__ int class_of(uint64_t key) { return (int)((1u << kIndexBits) - 1 - (unsigned)(key & ((1u << kIndexBits) - 1))); }
__device__ __forceinline__ uint64_t key_max(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ uint64_t key_min(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ uint64_t shuffled(uint64_t v, int mask)
{
    return ((uint64_t)(unsigned)__shfl_xor((int)(v >> 32), mask, 64) << 32) | (unsigned)__shfl_xor((int)v, mask, 64);
}
// The same order for less, where NaN is 0x7FC00000: the logit's bits are a double's upper half, whose sign and magnitude order as a float's do, and the class
// makes it larger the lower it is.
constexpr uint64_t kBelowAll = UINT64_C(0xFFF0000000000000);  // the double -inf: a place that nothing took
__device__ __forceinline__ uint64_t double_of(float x, int j)
{
    const unsigned b = __float_as_uint(x + 0.0f);
    return ((uint64_t)b << 32) | (unsigned)~(j ^ ((int)b >> 31));
}
__device__ __forceinline__ float logit_of_double(uint64_t d) { return d == kBelowAll ? -infinity() : __uint_as_float((unsigned)(d >> 32)); }
__device__ __forceinline__ int class_of_double(uint64_t d) { return ~((int)(unsigned)d ^ ((int)(unsigned)(d >> 32) >> 31)); }
constexpr int round_up(int n) { return n <= 1 ? 1 : 2 * round_up((n + 1) / 2); }  // to a power of two

template <int CTRL>
__device__ __forceinline__ uint64_t moved_key(uint64_t v)
{
    return ((uint64_t)moved<CTRL>((unsigned)(v >> 32)) << 32) | moved<CTRL>((unsigned)v);
}

// What a row's numbers come to.  m: the largest logit, total: the sum of exp(s (x - m)), weighted: the sum of s (x - m) times that.
struct RowSums {
    float m, total, weighted;
    __device__ __forceinline__ bool none() const { return total == 0.0f; }  // (every logit is -inf)
    __device__ __forceinline__ float log_total() const { return none() ? 0.0f : logf(total); }
    __device__ __forceinline__ float entropy() const { return none() ? 0.0f : logf(total) - weighted / total; }
};
__device__ __forceinline__ float base_of(float m) { return m == -infinity() ? 0.0f : m; }
// Half of a logit's distance from the largest, which whole may be beyond fp32 where s times it is not (the same bits, but for the scale)
__device__ __forceinline__ float half_distance(float x, float base) { return 0.5f * x - 0.5f * base; }

// The sums of a row from those of its parts, one in each lane of a team of W, in every lane.  A part's are of exp(s (x - its own largest)): with
// z = s (its largest - the row's), exp(z) times them, and z exp(z) times the total more of the weighted one.  A part of classes that are ruled out adds
// nothing: it has no largest to take z from (the distance of 0 to a row of the type's lowest values, times s, is infinite).
template <int W>
__device__ __forceinline__ RowSums joined(const RowSums& part, float scale)
{
    RowSums s;
    s.m = team_largest<W>(part.m);
    const float z = part.none() ? 0.0f : (base_of(part.m) - base_of(s.m)) * scale, f = part.none() ? 0.0f : __builtin_amdgcn_exp2f(z * kLog2e);
    s.total = team_sum<W>(f * part.total);
    s.weighted = team_sum<W>(f * (part.weighted + larger(z, -1e4f) * part.total));
    return s;
}

__device__ __forceinline__ void write_top(const AnswerArgs& a, int64_t row, int place, float x, int j, float base, float log_total)
{
    const bool none = x == -infinity();
    a.top_index[row * a.k + place] = none ? -1 : j;
    a.top_logp[row * a.k + place] = none ? -infinity() : half_distance(x, base) * (2.0f * a.scale) - log_total;
}
__device__ __forceinline__ void write_top(const AnswerArgs& a, int64_t row, int place, uint64_t key, float base, float log_total)
{
    write_top(a, row, place, key ? logit_of(key) : -infinity(), key ? class_of(key) : -1, base, log_total);
}
__device__ __forceinline__ void write_row(const AnswerArgs& a, int64_t row, int64_t token, float logit, float base, const RowSums& s)
{
    const float l = s.log_total();
    if (a.logp) a.logp[row] = token >= 0 && token < a.C ? half_distance(logit, base) * (2.0f * a.scale) - l : 0.0f;
    if (a.entropy) a.entropy[row] = s.entropy();
    if (a.stats) a.stats[2 * row] = base, a.stats[2 * row + 1] = l;
}

__device__ __forceinline__ float largest_of(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// y = c (x - base) in one instruction, c x + k with k = -c base rounded: every y of a row is off by the same `shift`, which is taken off its sums.
// (Where that rounding is no small number, x - base and then the product.)
struct Exponent {
    float base, c, k, shift, back;
    bool far;
    __device__ __forceinline__ Exponent(float base_, float c_) : base(base_), c(c_)
    {
        k = -(base * c);
        far = !(fabsf(k) < 65536.0f);
        shift = fmaf(base, c, k);
        back = __builtin_amdgcn_exp2f(-shift);
    }
};

// A row's part in a team's registers, as it is stored: vector t = v * TPR + lane starts at column t * VEC, the last one is moved back to end with the
// part; what it repeats and what no vector holds is -inf.  (Teams within a wavefront take as few vectors as hold a row, so only the last can be such.)
template <typename T, int VEC, int NV, int TPR>
struct Row {
    typename Vec<T, VEC>::type raw[NV];

    static __device__ __forceinline__ unsigned column(int v, int lane, int len, int nvec) { return (unsigned)min(min(v * TPR + lane, nvec - 1) * VEC, len - VEC); }
    __device__ __forceinline__ float at(int v, int i) const { return element<T, VEC>(raw[v], i); }
    __device__ __forceinline__ void load(const T* x, int len, int nvec, int lane)
    {
#pragma unroll
        for (int v = 0; v < NV; ++v) raw[v] = *reinterpret_cast<const typename Vec<T, VEC>::type*>(x + column(v, lane, len, nvec));
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (TPR < 64 && VEC > 1 && v < (NV <= 4 ? NV - 1 : NV - 2)) continue;
            if (TPR >= 64 && __builtin_amdgcn_readfirstlane(v * TPR + (int)(lane & ~63)) + 64 < nvec) continue;
            const int t = v * TPR + lane, first = t < nvec ? t * VEC - column(v, lane, len, nvec) : VEC;
            const T none = narrow<T>(-__builtin_inff());
            if constexpr (VEC == 1) {
                if (first > 0) raw[v] = none;
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (i < first) raw[v][i] = none;
            }
        }
    }
    // Between passes over a row in bf16: the compiler would keep its elements widened, in twice the registers.
    __device__ __forceinline__ void as_stored()
    {
        if constexpr (sizeof(T) == 2 && VEC == 8) {
            typedef unsigned Quad __attribute__((ext_vector_type(4)));
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                Quad q = __builtin_bit_cast(Quad, raw[v]);
                asm volatile("" : "+v"(q));
                raw[v] = __builtin_bit_cast(typename Vec<T, VEC>::type, q);
            }
        }
    }
    // Every NaN in the one form that double_of takes.
    __device__ __forceinline__ void one_nan()
    {
        const T nan = narrow<T>(__uint_as_float(0x7FC00000u));
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if constexpr (VEC == 1) {
                if (at(v, 0) != at(v, 0)) raw[v] = nan;
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (at(v, i) != at(v, i)) raw[v][i] = nan;
            }
        }
    }
    // The largest of this lane's elements; a row with a NaN is told by its sum.
    __device__ __forceinline__ float largest() const
    {
        float m = -__builtin_inff();
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if constexpr (VEC == 1) {
                m = larger(m, at(v, 0));
            } else {
#pragma unroll
                for (int i = 0; i < VEC; i += 2) m = largest_of(m, at(v, i), at(v, i + 1));
            }
        }
        return m;
    }
    // The largest of each fourth of this lane's elements.
    __device__ __forceinline__ void largest_four(float (&m)[4]) const
    {
#pragma unroll
        for (int q = 0; q < 4; ++q) m[q] = -__builtin_inff();
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < VEC; ++i) m[i & 3] = larger(m[i & 3], at(v, i));
    }
    template <typename Y>
    __device__ __forceinline__ void add_up(Y exponent, float& total, float& weighted)
    {
        as_stored();
        total = weighted = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float y = exponent(at(v, i)), p = __builtin_amdgcn_exp2f(y);
                total += p;
                weighted += p * larger(y, -1e4f);  // (p is 0 there)
            }
    }
    // the sums of 2^y and y 2^y over this lane's elements, y = c (x - base)
    __device__ __forceinline__ void sums(const Exponent& e, float& total, float& weighted)
    {
        if (!e.far) {
            add_up([&](float x) { return fmaf(x, e.c, e.k); }, total, weighted);
            weighted = (weighted - e.shift * total) * e.back, total *= e.back;
        } else {
            add_up([&](float x) { return (x - e.base) * e.c; }, total, weighted);
        }
    }
};

// Sorted lists of keys in a lane's registers, largest first; lengths are powers of two.
__device__ __forceinline__ void in_order(uint64_t& a, uint64_t& b)
{
    const uint64_t low = key_min(a, b);
    a = key_max(a, b);
    b = low;
}
// Places LO, LO + R, LO + 2 R ... of N: two sorted halves become one list (odd-even merging, K. E. Batcher 1968).
template <int LO, int N, int R, int L>
__device__ __forceinline__ void merge_halves(uint64_t (&list)[L])
{
    if constexpr (2 * R < N) {
        merge_halves<LO, N, 2 * R>(list);
        merge_halves<LO + R, N, 2 * R>(list);
#pragma unroll
        for (int i = LO + R; i + R < LO + N; i += 2 * R) in_order(list[i], list[i + R]);
    } else {
        in_order(list[LO], list[LO + R]);
    }
}
template <int LO, int N, int L>
__device__ __forceinline__ void sort_list(uint64_t (&list)[L])
{
    if constexpr (N > 1) {
        sort_list<LO, N / 2>(list);
        sort_list<LO + N / 2, N / 2>(list);
        merge_halves<LO, N, 1>(list);
    }
}
// A list that first falls and then rises is put in order.
template <int L>
__device__ __forceinline__ void straighten(uint64_t (&list)[L])
{
    if constexpr (L > 1) {
#pragma unroll
        for (int n = 0; n < L / 2; ++n) in_order(list[n], list[n + L / 2]);
        if constexpr (L > 2) {
#pragma unroll
            for (int n = 0; n < L / 2; ++n) in_order(list[n / (L / 4) * (L / 2) + n % (L / 4)], list[n / (L / 4) * (L / 2) + n % (L / 4) + L / 4]);
        }
        if constexpr (L > 4) {
#pragma unroll
            for (int n = 0; n < L / 2; ++n) in_order(list[n / (L / 8) * (L / 4) + n % (L / 8)], list[n / (L / 8) * (L / 4) + n % (L / 8) + L / 8]);
        }
        if constexpr (L > 8) {
#pragma unroll
            for (int n = 0; n < L / 2; ++n) in_order(list[n / (L / 16) * (L / 8) + n % (L / 16)], list[n / (L / 16) * (L / 8) + n % (L / 16) + L / 16]);
        }
        if constexpr (L > 16) {
#pragma unroll
            for (int n = 0; n < L / 2; ++n) in_order(list[n / (L / 32) * (L / 16) + n % (L / 32)], list[n / (L / 32) * (L / 16) + n % (L / 32) + L / 32]);
        }
        if constexpr (L > 32) {
#pragma unroll
            for (int n = 0; n < L / 2; ++n) in_order(list[n / (L / 64) * (L / 32) + n % (L / 64)], list[n / (L / 64) * (L / 32) + n % (L / 64) + L / 64]);
        }
    }
}
template <int W>
__device__ __forceinline__ uint64_t from_other(uint64_t v)  // that of the lane W away, or of one that holds the same
{
    if constexpr (W == 1) return moved_key<0xB1>(v);
    else if constexpr (W == 2) return moved_key<0x4E>(v);
    else if constexpr (W == 4) return moved_key<0x141>(v);
    else if constexpr (W == 8) return moved_key<0x140>(v);
    else return shuffled(v, W);
}
// The K largest of a team's sorted lists of L, from lanes W away on: lists are put together until they have K places, from then on the larger of places
// crosswise are the K largest of both.
template <int K, int TPR, int W, int L>
__device__ __forceinline__ void team_list(const uint64_t (&list)[L], uint64_t (&top)[K])
{
    if constexpr (W >= TPR) {
#pragma unroll
        for (int i = 0; i < K; ++i) top[i] = i < L ? list[i] : kBelowAll;
    } else if constexpr (2 * L <= K) {
        uint64_t both[2 * L];
#pragma unroll
        for (int i = 0; i < L; ++i) both[i] = list[i], both[2 * L - 1 - i] = from_other<W>(list[i]);
        straighten(both);
        team_list<K, TPR, 2 * W>(both, top);
    } else {
        uint64_t both[L];
#pragma unroll
        for (int i = 0; i < L; ++i) both[i] = key_max(list[i], from_other<W>(list[L - 1 - i]));
        straighten(both);
        team_list<K, TPR, 2 * W>(both, top);
    }
}

// The same number, of which the compiler knows nothing: what is worked out from it stays where it is needed, and is not kept in registers from one
// row to the next (75 instead of 106 for rows of 32,768 in bf16, so that a compute unit has three workgroups of 512 and not two: answers 73 us and not 89).
__device__ __forceinline__ int opaque(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// ---- answers, rows of part of a wavefront ------------------------------------------------------------------------

// KT: places of a lane's list, as many as are asked for or as there are classes (0: no alternatives)
template <typename T, int VEC, int NV, int TPR, int KT>
__global__ __launch_bounds__(256) void gp_answer_short(AnswerArgs a)
{
    constexpr int TEAMS = 256 / TPR;
    for (int64_t row = (int64_t)blockIdx.x * TEAMS + threadIdx.x / TPR; row < a.N; row += (int64_t)gridDim.x * TEAMS) {
        const int lane = opaque(threadIdx.x % TPR);
        const T* const x = (const T*)a.x + row * a.ld;
        const int64_t token = a.logp ? token_at(a.tokens, a.wide, row) : -1;
        Row<T, VEC, NV, TPR> e;
        e.load(x, a.C, a.nvec, lane);
        const float logit = token >= 0 && token < a.C ? widen(x[token]) : 0.0f;
        RowSums s;
        s.m = base_of(team_largest<TPR>(e.largest()));
        float total, weighted;
        e.sums(Exponent(s.m, a.scale * kLog2e), total, weighted);
        s.total = team_sum<TPR>(total), s.weighted = team_sum<TPR>(weighted) * kLn2;
        if (lane == 0) write_row(a, row, token, logit, s.m, s);
        if constexpr (KT > 0) {
            if (s.total != s.total) e.one_nan();
            // this lane's elements in stretches of KT or fewer, sorted and merged
            constexpr int E = NV * VEC, L = KT < round_up(E) ? KT : round_up(E);
            uint64_t mine[L], list[KT];
#pragma unroll
            for (int first = 0; first < E; first += L) {
                uint64_t part[L];
#pragma unroll
                for (int n = 0; n < L; ++n) {
                    const int v = min(first + n, E - 1) / VEC, i = min(first + n, E - 1) % VEC;
                    part[n] = first + n < E ? double_of(e.at(v, i), e.column(v, lane, a.C, a.nvec) + i) : kBelowAll;
                }
                sort_list<0, L>(part);
                if (first == 0) {
#pragma unroll
                    for (int n = 0; n < L; ++n) mine[n] = part[n];
                } else {
#pragma unroll
                    for (int n = 0; n < L; ++n) mine[n] = key_max(mine[n], part[L - 1 - n]);
                    straighten(mine);
                }
            }
            team_list<KT, TPR, 1>(mine, list);
            const float l = s.log_total();
            constexpr int MINE = (KT + TPR - 1) / TPR;
            uint64_t d[MINE] = {};
#pragma unroll
            for (int i = 0; i < KT; ++i) d[i / TPR] = lane == i % TPR ? list[i] : d[i / TPR];
#pragma unroll
            for (int i = 0; i < MINE; ++i)
                if (i * TPR + lane < a.k) write_top(a, row, i * TPR + lane, logit_of_double(d[i]), class_of_double(d[i]), s.m, l);
            for (int place = KT + lane; place < a.k; place += TPR) write_top(a, row, place, -infinity(), 0, s.m, l);  // (there are KT classes or fewer)
        }
    }
}

// ---- answers, rows of a wavefront or a workgroup ----------------------------------------------------------------

template <int TPR>
__device__ __forceinline__ void team_barrier()
{
    if constexpr (TPR > 64) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// What a team shares in LDS.
template <int TPR>
struct TeamLds {
    static constexpr int WAVES = TPR / 64, ROOM = TPR > 64 ? kRoom : kRoom / 4;
    RowSums sums[WAVES];
    float group[TPR > 64 ? 256 : 1];
    float bound;
    int count;
    uint64_t best[WAVES];
    uint64_t list[ROOM + 8];
};

__device__ __forceinline__ unsigned ordered(float x)
{
    const unsigned b = __float_as_uint(x);
    return b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
}
// The k-th largest of a wavefront's 64 values (k <= 64), in every lane: few by taking the largest away, many by counting.
__device__ __forceinline__ float kth_largest(float v, int k)
{
    if (k <= 16) {
        float last = infinity();
        for (int r = 0; r < k; ++r) {
            last = team_largest<64>(v);
            const uint64_t with = __ballot(v == last);
            if ((int)(threadIdx.x & 63) == __ffsll((unsigned long long)with) - 1) v = -infinity();
        }
        return last;
    }
    int above = 0;
    for (int l = 0; l < 64; ++l) above += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l)) > v;
    return -team_largest<64>(above < k ? -v : -infinity());
}
// A bound that k or more of a wavefront's 256 values reach, and few others: the k-th largest to its first 16 bits, found bit by bit (0: fewer than k are there).
__device__ __forceinline__ unsigned kth_bound(const unsigned (&v)[4], int k)
{
    unsigned t = 0;
    for (int bit = 31; bit >= 16; --bit) {
        const unsigned with = t | 1u << bit;
        int n = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) n += __popcll(__ballot(v[q] >= with));
        if (n >= k) t = with;
    }
    return t;
}
// As a float to compare with: what is not below it, and NaN, which is above everything, is not less.
__device__ __forceinline__ float bound_of(unsigned t) { return __uint_as_float(t & 0x80000000u ? t & 0x7FFFFFFFu : ~t); }

// How many of `count` keys in LDS are larger than `key`; eight reads are under way at a time, `list` has eight places more.
__device__ __forceinline__ int rank_of(const uint64_t* list, int count, uint64_t key)
{
    int rank = 0;
    for (int j = 0; j < count; j += 8) {
        uint64_t other[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) other[u] = list[j + u];
#pragma unroll
        for (int u = 0; u < 8; ++u) rank += j + u < count && other[u] > key;
    }
    return rank;
}

// Where the largest key of all is in `best` of every lane.
template <int TPR>
__device__ __forceinline__ uint64_t team_best(uint64_t best, TeamLds<TPR>& lds)
{
#pragma unroll
    for (int w = 1; w < 64; w *= 2) best = key_max(best, shuffled(best, w));
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) lds.best[threadIdx.x >> 6] = best;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < TPR / 64; ++w) best = key_max(best, lds.best[w]);
        __syncthreads();
    }
    return best;
}

// One team to a row, or to a row's part.  TPR 64: four rows to a workgroup.
template <typename T, int VEC, int NV, int TPR>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void gp_answer_rows(AnswerArgs a)
{
    constexpr int BLOCK = TPR < 256 ? 256 : TPR, TEAMS = BLOCK / TPR;
    __shared__ TeamLds<TPR> all_lds[TEAMS];
    TeamLds<TPR>& lds = all_lds[threadIdx.x / TPR];
    const int wave = threadIdx.x % TPR >> 6;
    const int64_t items = a.N * a.parts;
    for (int64_t item = (int64_t)blockIdx.x * TEAMS + (TEAMS > 1 ? threadIdx.x / TPR : 0); item < items; item += (int64_t)gridDim.x * TEAMS) {
        const int lane = opaque(threadIdx.x % TPR);
        const int64_t row = a.parts == 1 ? item : item / a.parts;
        const int part = a.parts == 1 ? 0 : (int)(item - row * a.parts);
        const int lo = (int)((int64_t)a.nvec * part / a.parts), hi = (int)((int64_t)a.nvec * (part + 1) / a.parts);
        const int off = lo * VEC, len = min(hi * VEC, a.C) - off;
        const T* const x = (const T*)a.x + row * a.ld;
        const int64_t token = a.logp && a.parts == 1 ? token_at(a.tokens, a.wide, row) : -1;
        Row<T, VEC, NV, TPR> e;
        e.load(x + off, len, hi - lo, lane);
        const float logit = token >= 0 && token < a.C ? widen(x[token]) : 0.0f;
        // every wavefront takes its own largest as the base of its sums, which are joined afterwards
        const float mine = e.largest();
        RowSums s;
        s.m = team_largest<64>(mine);
        e.sums(Exponent(base_of(s.m), a.scale * kLog2e), s.total, s.weighted);
        e.as_stored();
        s.total = team_sum<64>(s.total), s.weighted = team_sum<64>(s.weighted) * kLn2;
        float bound = -infinity();
        if (lane == 0) lds.count = 0;
        if constexpr (TPR > 64) {
            // the largest of 64 groups of lanes, or of 256
            const bool many = a.k > kFewTop;
            const float pair = team_largest<TPR / 256>(mine), group = many ? pair : team_largest<TPR / 64>(mine);
            const int lanes = many ? TPR / 256 : TPR / 64;
            if ((lane & (lanes - 1)) == 0) lds.group[lane / lanes] = group;
            if ((lane & 63) == 0) lds.sums[wave] = s;
            __syncthreads();
            s = joined<TPR / 64>(lds.sums[lane & (TPR / 64 - 1)], a.scale);
            if (a.k > 0) {
                if (wave == 0) {
                    if (many) {
                        const unsigned v[4] = {ordered(lds.group[lane]), ordered(lds.group[lane + 64]), ordered(lds.group[lane + 128]), ordered(lds.group[lane + 192])};
                        bound = bound_of(kth_bound(v, a.k));
                    } else {
                        bound = kth_largest(lds.group[lane], a.k);
                    }
                    if (lane == 0) lds.bound = bound;
                }
                __syncthreads();
                bound = lds.bound;
            }
        } else if (a.k > kFewTop) {
            float four[4];
            e.largest_four(four);
            const unsigned v[4] = {ordered(four[0]), ordered(four[1]), ordered(four[2]), ordered(four[3])};
            bound = bound_of(kth_bound(v, a.k));
        } else if (a.k > 0) {
            bound = kth_largest(mine, a.k);
        }
        const float base = base_of(s.m);
        if (lane == 0) {
            if (a.parts == 1) {
                write_row(a, row, token, logit, base, s);
            } else {
                float* const to = a.partial + 4 * item;
                to[0] = s.m, to[1] = s.total, to[2] = s.weighted;
            }
        }
        if (a.k > 0) {
            // whatever is not below the bound; -inf is no alternative, NaN above all
            const auto offer = [&](float y, int j) {
                if (!(y < bound) && y != -infinity()) {
                    const int at = atomicAdd(&lds.count, 1);
                    if (at < TeamLds<TPR>::ROOM) lds.list[at] = key_of(y, j);
                }
            };
            const bool some = !(mine < bound) || s.total != s.total;
            uint64_t with = __ballot(some);
            if (TPR > 64 && NV * VEC >= 32 && __popcll(with) <= 4) {
                // few of a wavefront's lanes have one: all lanes look at a lane's elements, one each, as they are in memory (64 elements of every lane looked at
                // by all took 300 of 930 instructions: 3,764 x 17,000 in bf16, five best 57 -> 49 us; of 8 elements less than the reads: 160 -> 184)
                const int n = opaque(lane) & 63, v = n / VEC, i = n % VEC;
                for (; with != 0; with &= with - 1) {
                    const int from = (threadIdx.x & ~63) + __ffsll((unsigned long long)with) - 1, t = v * TPR + from;
                    const int col = (int)e.column(v, from, len, hi - lo);
                    if (n < NV * VEC && t < hi - lo && i >= t * VEC - col) offer(widen(x[off + col + i]), off + col + i);
                }
            } else if (some) {
                const int here = opaque(lane);
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) offer(e.at(v, i), off + (int)e.column(v, here, len, hi - lo) + i);
            }
            team_barrier<TPR>();
            const int count = __builtin_amdgcn_readfirstlane(lds.count);
            const float l = s.log_total();
            uint64_t* const keys = a.parts == 1 ? nullptr : a.keys + row * a.parts * a.k + part;  // place by place, in each the parts side by side
            if (count <= TeamLds<TPR>::ROOM) {
                for (int c = lane; c < count; c += TPR) {
                    const uint64_t key = lds.list[c];
                    const int rank = rank_of(lds.list, count, key);
                    if (rank < a.k) {
                        if (keys)
                            keys[(int64_t)rank * a.parts] = key;
                        else
                            write_top(a, row, rank, key, base, l);
                    }
                }
                for (int place = count + lane; place < a.k; place += TPR) {
                    if (keys)
                        keys[(int64_t)place * a.parts] = 0;
                    else
                        write_top(a, row, place, 0, base, l);
                }
            } else {
                uint64_t last = UINT64_C(1) << 60;  // (above every key)
                for (int place = 0; place < a.k; ++place) {
                    uint64_t best = 0;
                    for (int j = lane; j < len; j += TPR) {  // (as it is in memory: what is rare shall cost others no registers)
                        const float y = widen(x[off + j]);
                        const uint64_t key = y != -infinity() ? key_of(y, off + j) : 0;
                        if (key < last && key > best) best = key;
                    }
                    last = team_best<TPR>(best, lds);
                    if (lane == 0) {
                        if (keys)
                            keys[(int64_t)place * a.parts] = last;
                        else
                            write_top(a, row, place, last, base, l);
                    }
                }
            }
        }
        team_barrier<TPR>();  // (the next row's numbers go where this one's were)
    }
}

// The sums of a row's parts, in every lane of a wavefront.
__device__ __forceinline__ RowSums join_parts(const float* partial, int parts, int lane, int lanes, float scale)
{
    RowSums s{-infinity(), 0.0f, 0.0f};
    for (int p = lane; p < parts; p += lanes) {
        const float4 q = *(const float4*)(partial + 4 * (int64_t)p);
        const float m = larger(s.m, q.x);  // (as in `joined`: no distance where nothing is)
        const float z = s.total == 0.0f ? 0.0f : (base_of(s.m) - base_of(m)) * scale, y = q.y == 0.0f ? 0.0f : (base_of(q.x) - base_of(m)) * scale;
        const float f = s.total == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(z * kLog2e), g = q.y == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(y * kLog2e);
        s.weighted = f * (s.weighted + larger(z, -1e4f) * s.total) + g * (q.z + larger(y, -1e4f) * q.y);
        s.total = f * s.total + g * q.y;
        s.m = m;
    }
    return joined<64>(s, scale);
}

// Joins the parts of a row: its sums, and the largest of the parts' keys by the same bound as above, of 256 groups (place by place, so that each has
// keys of every rank).  A wavefront for few keys, a workgroup of 1,024 for many (one row of 190 parts by 20 keys 5 us; by 256 lanes 14).
template <typename T, int LANES>
__global__ __launch_bounds__(LANES) void gp_answer_join(AnswerArgs a)
{
    constexpr int WAVES = LANES / 64;
    __shared__ uint64_t list[kRoom + 8], best_at[WAVES];
    __shared__ unsigned group[256], bound_at;
    __shared__ RowSums sums[WAVES];
    __shared__ int count;
    const int lane = threadIdx.x;
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const uint64_t* const keys = a.keys + row * a.parts * a.k;
        const int all = a.parts * a.k;
        const int64_t token = a.logp ? token_at(a.tokens, a.wide, row) : -1;
        constexpr int OWN = 4;  // keys that a lane holds; what is beyond is read twice
        uint64_t own[OWN], mine = 0;
#pragma unroll
        for (int i = 0; i < OWN; ++i) own[i] = i * LANES + lane < all ? keys[i * LANES + lane] : 0;
        const float logit = token >= 0 && token < a.C ? widen(((const T*)a.x)[row * a.ld + token]) : 0.0f;
        RowSums s = join_parts(a.partial + 4 * row * a.parts, a.parts, lane, LANES, a.scale);
#pragma unroll
        for (int i = 0; i < OWN; ++i) mine = key_max(mine, own[i]);
        for (int j = OWN * LANES + lane; j < all; j += LANES) mine = key_max(mine, keys[j]);
        // (logits alone decide the bound: a key's upper part)
        if constexpr (WAVES > 1) {
            const unsigned o = (unsigned)(mine >> kIndexBits), p = max(o, moved<0xB1>(o)), q = max(p, moved<0x4E>(p));
            if ((lane & 3) == 0) group[lane >> 2] = q;
            if ((lane & 63) == 0) sums[lane >> 6] = s;
        }
        if (lane == 0) count = 0;
        __syncthreads();
        if constexpr (WAVES > 1) s = joined<WAVES>(sums[lane & (WAVES - 1)], a.scale);
        const float base = base_of(s.m);
        if (lane == 0) write_row(a, row, token, logit, base, s);
        if (a.k > 0) {
            if (lane < 64) {
                unsigned v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = WAVES > 1 ? group[lane + 64 * i] : (unsigned)(own[i] >> kIndexBits);
                const unsigned t = kth_bound(v, a.k);
                if (lane == 0) bound_at = t;
            }
            __syncthreads();
            const unsigned bound = bound_at;
            const auto offer = [&](uint64_t key) {
                if ((unsigned)(key >> kIndexBits) >= bound && key > 0) {
                    const int at = atomicAdd(&count, 1);
                    if (at < kRoom) list[at] = key;
                }
            };
#pragma unroll
            for (int i = 0; i < OWN; ++i) offer(own[i]);
            for (int j = OWN * LANES + lane; j < all; j += LANES) offer(keys[j]);
            __syncthreads();
            const float l = s.log_total();
            const int found = __builtin_amdgcn_readfirstlane(count);
            if (found <= kRoom) {
                for (int c = lane; c < found; c += LANES) {
                    const uint64_t key = list[c];
                    const int rank = rank_of(list, found, key);
                    if (rank < a.k) write_top(a, row, rank, key, base, l);
                }
                for (int place = found + lane; place < a.k; place += LANES) write_top(a, row, place, 0, base, l);
            } else {
                uint64_t last = UINT64_C(1) << 60;  // (above every key)
                for (int place = 0; place < a.k; ++place) {
                    uint64_t best = 0;
                    for (int j = lane; j < all; j += LANES) {
                        const uint64_t key = keys[j];
                        if (key < last && key > best) best = key;
                    }
#pragma unroll
                    for (int w = 1; w < 64; w *= 2) best = key_max(best, shuffled(best, w));
                    if ((lane & 63) == 0) best_at[lane >> 6] = best;
                    __syncthreads();
                    last = 0;
#pragma unroll
                    for (int w = 0; w < WAVES; ++w) last = key_max(last, best_at[w]);
                    if (lane == 0) write_top(a, row, place, last, base, l);
                    __syncthreads();
                }
            }
        }
        __syncthreads();
    }
}

// ---- gradient of answers -----------------------------------------------------------------------------------------

struct AnswerGradArgs {
    const void* x;
    int64_t ld, N;
    int C, nvec;
    const void* tokens;
    int wide;
    float scale;
    const float *stats, *entropy, *g1, *g2;
    int64_t s1, s2;  // distances of g1's and g2's elements: 0 or 1
    void* grad;
    int64_t ldg;
};

// One vector per thread and step.  A row's last vector is moved back to end with the row (what it repeats is written twice, identically).
template <typename T, int VEC>
__global__ __launch_bounds__(256) void gp_answer_grad(AnswerGradArgs a)
{
    constexpr int U = 2;
    const int64_t total = a.N * a.nvec;
    for (int64_t b0 = (int64_t)blockIdx.x * (U * 256); b0 < total; b0 += (int64_t)gridDim.x * (U * 256)) {
        const int64_t r0 = b0 / a.nvec;
        const unsigned rem = (unsigned)(b0 - r0 * a.nvec);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const unsigned place = rem + u * 256 + threadIdx.x, q = place / (unsigned)a.nvec;
            const int64_t row = r0 + q;
            if (row >= a.N) continue;
            const int col = min((int)(place - q * a.nvec) * VEC, a.C - VEC);
            float v[VEC];
            load_vec<T, VEC>((const T*)a.x + row * a.ld + col, v);
            const int64_t token = a.g1 ? token_at(a.tokens, a.wide, row) : -1;
            const bool named = token >= 0 && token < a.C;
            const float base = a.stats[2 * row], l = a.stats[2 * row + 1];
            const float g1 = named ? a.g1[row * a.s1] * a.scale : 0.0f, g2 = a.g2 ? a.g2[row * a.s2] * a.scale : 0.0f, h = a.g2 ? a.entropy[row] : 0.0f;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float logp = (v[i] - base) * a.scale - l, p = __builtin_amdgcn_exp2f(logp * kLog2e);
                v[i] = (named && token == col + i ? g1 : 0.0f) - p * (g1 + g2 * (larger(logp, -1e4f) + h));
            }
            store_vec<T, VEC>((T*)a.grad + row * a.ldg + col, v);
        }
    }
}

// ---- distillation ----------------------------------------------------------------------------------------------------

struct DistillArgs {
    const void* x;
    int64_t ld, N;
    int C, nvec;
    const void* index;
    int wide;
    int64_t ldi;
    const void* teacher;
    int64_t ldv;
    int wide_teacher;  // fp32
    int K;
    float T;
    float *loss, *stats;
    const float* from;  // stats that an earlier pass left: no loss, the gradient alone
    const float* g;
    int64_t sg;
    void* grad;
    int64_t ldg;
    int parts;
    float* partial;
};

__device__ __forceinline__ int64_t entry_index(const DistillArgs& a, int64_t row, int k)
{
    return token_at(a.index, a.wide, row * a.ldi + k);
}
__device__ __forceinline__ float entry_logit(const DistillArgs& a, int64_t row, int k)
{
    return a.wide_teacher ? ((const float*)a.teacher)[row * a.ldv + k] : widen(((const bf16_t*)a.teacher)[row * a.ldv + k]);
}

// Entries of a row's teacher, PER of them in a lane of a team of W: k = lane * PER + i.
template <int W, int PER>
struct Teacher {
    int at[PER];    // the class, -1: none
    float q[PER], logq[PER], logit[PER];  // its probability, the log of it, the student's logit
    bool some;      // the row has an entry that counts

    template <typename T>
    __device__ __forceinline__ void load(const DistillArgs& a, int64_t row, const T* x, int lane)
    {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int k = lane * PER + i;
            const int64_t j = k < a.K ? entry_index(a, row, k) : -1;
            at[i] = j >= 0 && j < a.C ? (int)j : -1;
            q[i] = at[i] >= 0 ? entry_logit(a, row, k) : -infinity();
            logit[i] = at[i] >= 0 ? widen(x[at[i]]) : 0.0f;
        }
    }
    __device__ __forceinline__ void weigh(float T)
    {
        float m = -infinity(), total = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) m = larger(m, q[i]);
        m = base_of(team_largest<W>(m));
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            logq[i] = (q[i] - m) / T;
            q[i] = __builtin_amdgcn_exp2f(logq[i] * kLog2e);
            total += q[i];
        }
        total = team_sum<W>(total);
        some = !(total == 0.0f);
        const float l = some ? logf(total) : 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            logq[i] -= l;
            q[i] = some ? q[i] / total : 0.0f;
        }
    }
    // T^2 q (log q - log p) as 4 T q (T (log q + log(sum)) - (logit - base)) / 4, in quarters: (logit - base) / T may be beyond fp32 where the loss is not (a class at the
    // type's lowest value, T below 1), and so may logit - base and a sum of such
    __device__ __forceinline__ float loss(float T, float base, float log_total) const
    {
        const float t = 0.25f * T, b = 0.25f * base;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (!(q[i] == 0.0f)) sum += q[i] * (t * (logq[i] + log_total) - (0.25f * logit[i] - b));
        return 4.0f * T * team_sum<W>(sum);
    }
};

// Rows of part of a wavefront: the gradient goes through LDS, where the entries' shares are taken off, one after another, and leaves it in whole vectors (single
// stores of a last vector's elements took 6 us of 66).  What is left above the bytes' time is waiting: 507,001 x 47, 390 instructions of the vector
// unit a wavefront, 20 us of 57, and 9 us of a wavefront's life.  Asking for the next row ahead, with workgroups that walk, took longer (70 us), walking alone too (65).
template <typename T, int VEC, int NV, int TPR, int PER>
__global__ __launch_bounds__(256) void gp_distill_short(DistillArgs a)
{
    constexpr int TEAMS = 256 / TPR, CELLS = NV * VEC * TPR;
    __shared__ __attribute__((aligned(16))) float cells[TEAMS][CELLS];
    float* const mine = cells[threadIdx.x / TPR];
    const float c = kLog2e / a.T;
    for (int64_t row = (int64_t)blockIdx.x * TEAMS + threadIdx.x / TPR; row < a.N; row += (int64_t)gridDim.x * TEAMS) {
        const int lane = opaque(threadIdx.x % TPR);
        const T* const x = (const T*)a.x + row * a.ld;
        Row<T, VEC, NV, TPR> e;
        Teacher<TPR, PER> t;
        e.load(x, a.C, a.nvec, lane);
        t.load(a, row, x, lane);
        float base, log_total;
        if (a.from) {
            base = a.from[2 * row], log_total = a.from[2 * row + 1];
        } else {
            float total, weighted;
            base = base_of(team_largest<TPR>(e.largest()));
            e.sums(Exponent(base, c), total, weighted);
            total = team_sum<TPR>(total);
            log_total = total == 0.0f ? 0.0f : logf(total);
        }
        t.weigh(a.T);
        if (!a.from) {
            const float loss = t.some ? t.loss(a.T, base, log_total) : 0.0f;
            if (lane == 0) {
                if (a.loss) a.loss[row] = loss;
                if (a.stats) a.stats[2 * row] = base, a.stats[2 * row + 1] = log_total;
            }
        }
        if (!a.grad) continue;
        const float f = a.g[row * a.sg] * a.T, l2 = log_total * kLog2e;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int at = v * TPR + lane, col = e.column(v, lane, a.C, a.nvec), first = at < a.nvec ? at * VEC - col : VEC;
            float y[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float p = __builtin_amdgcn_exp2f((e.at(v, i) - base) * c - l2);
                y[i] = t.some ? f * p : 0.0f;
            }
            if (v < NV - 1) {  // (whole)
#pragma unroll
                for (int i = 0; i < VEC; ++i) mine[at * VEC + i] = y[i];
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (i >= first) mine[col + i] = y[i];
            }
        }
        team_barrier<64>();
        // one lane of a team at a time, so that entries of one class go in their order: a wavefront's additions in LDS are done in the order of its
        // instructions, and the barrier keeps those of one turn ahead of the next one's (it is none but for the compiler, which might make one turn of all)
        for (int turn = 0; turn * PER < a.K; ++turn) {
            if (lane == turn) {
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (t.some && t.at[i] >= 0) atomicAdd(mine + t.at[i], -f * t.q[i]);  // (0 times an f that is no number is none)
            }
            team_barrier<64>();
        }
        T* const out = (T*)a.grad + row * a.ldg;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int at = v * TPR + lane, col = v < NV - 1 ? at * VEC : (int)e.column(v, lane, a.C, a.nvec);
            if (at >= a.nvec) continue;
            float y[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) y[i] = mine[col + i];
            store_vec<T, VEC>(out + col, y);
        }
    }
}

// Rows of a wavefront or a workgroup, or parts of them where `from` has their sums: the gradient is written from the registers, then the entries' classes once more.
template <typename T, int VEC, int NV, int TPR>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void gp_distill_rows(DistillArgs a)
{
    constexpr int BLOCK = TPR < 256 ? 256 : TPR, TEAMS = BLOCK / TPR, WAVES = TPR / 64;
    __shared__ RowSums lds[WAVES];
    __shared__ float some;
    const int wave = threadIdx.x % TPR >> 6;
    const int64_t items = a.N * a.parts;
    const float c = kLog2e / a.T;
    for (int64_t item = (int64_t)blockIdx.x * TEAMS + (TEAMS > 1 ? threadIdx.x / TPR : 0); item < items; item += (int64_t)gridDim.x * TEAMS) {
        const int lane = opaque(threadIdx.x % TPR);
        const int64_t row = a.parts == 1 ? item : item / a.parts;
        const int part = a.parts == 1 ? 0 : (int)(item - row * a.parts);
        const int lo = (int)((int64_t)a.nvec * part / a.parts), hi = (int)((int64_t)a.nvec * (part + 1) / a.parts);
        const int off = lo * VEC, len = min(hi * VEC, a.C) - off;
        const T* const x = (const T*)a.x + row * a.ld;
        Row<T, VEC, NV, TPR> e;
        e.load(x + off, len, hi - lo, lane);
        Teacher<64, 1> t;
        t.some = true;
        if (wave == 0) t.load(a, row, x, lane);
        float base, log_total;
        if (a.from) {
            base = a.from[2 * row], log_total = a.from[2 * row + 1];
        } else {
            RowSums sum;
            sum.m = team_largest<64>(e.largest());
            e.sums(Exponent(base_of(sum.m), c), sum.total, sum.weighted);
            e.as_stored();
            sum.total = team_sum<64>(sum.total);
            sum.weighted = 0.0f;
            if constexpr (TPR > 64) {
                if ((lane & 63) == 0) lds[wave] = sum;
                __syncthreads();
                sum = joined<WAVES>(lds[lane & (WAVES - 1)], 1.0f / a.T);
            }
            base = base_of(sum.m), log_total = sum.log_total();
        }
        if (wave == 0) {
            t.weigh(a.T);
            if (!a.from) {
                const float loss = t.some ? t.loss(a.T, base, log_total) : 0.0f;
                if (lane == 0) {
                    if (a.loss) a.loss[row] = loss;
                    if (a.stats) a.stats[2 * row] = base, a.stats[2 * row + 1] = log_total;
                }
            }
        }
        if (!a.grad) {
            if constexpr (TPR > 64) __syncthreads();
            continue;
        }
        if constexpr (TPR > 64) {
            if (lane == 0) some = t.some ? 1.0f : 0.0f;
            __syncthreads();
            t.some = some != 0.0f;
        }
        const float f = a.g[row * a.sg] * a.T, l2 = log_total * kLog2e;
        T* const out = (T*)a.grad + row * a.ldg;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int at = v * TPR + lane;
            if (at >= hi - lo) continue;
            const int col = off + e.column(v, lane, len, hi - lo), first = off + at * VEC - col;
            float y[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float p = __builtin_amdgcn_exp2f((e.at(v, i) - base) * c - l2);
                y[i] = t.some ? f * p : 0.0f;
            }
            if (first == 0) {
                store_vec<T, VEC>(out + col, y);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (i >= first) out[col + i] = narrow<T>(y[i]);
            }
        }
        team_barrier<TPR>();  // (a workgroup's stores to one place are seen in their order)
        if (wave == 0) {
            float taken = 0.0f;
            for (int k = 0; k < a.K; ++k) {
                const int at = __builtin_amdgcn_readlane(t.at[0], k);
                const float q = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(t.q[0]), k));
                if (at == t.at[0]) taken += q;
            }
            if (t.some && t.at[0] >= off && t.at[0] < off + len) {
                const float p = __builtin_amdgcn_exp2f((t.logit[0] - base) * c - l2);
                out[t.at[0]] = narrow<T>(f * (p - taken));
            }
        }
        if constexpr (TPR > 64) __syncthreads();
    }
}

// Joins the parts of a row: its sums, and the loss.
template <typename T>
__global__ __launch_bounds__(256) void gp_distill_join(DistillArgs a)
{
    for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < a.N; row += (int64_t)gridDim.x * 4) {
        const int lane = threadIdx.x & 63;
        Teacher<64, 1> t;
        t.load(a, row, (const T*)a.x + row * a.ld, lane);
        const RowSums s = join_parts(a.partial + 4 * row * a.parts, a.parts, lane, 64, 1.0f / a.T);
        t.weigh(a.T);
        const float base = base_of(s.m), l = s.log_total(), loss = t.some ? t.loss(a.T, base, l) : 0.0f;
        if (lane == 0) {
            if (a.loss) a.loss[row] = loss;
            if (a.stats) a.stats[2 * row] = base, a.stats[2 * row + 1] = l;
        }
    }
}

// ---- host ----------------------------------------------------------------------------------------------------------

constexpr int64_t kMaxBlocks = 1 << 20;  // of a launch; workgroups walk on through the rest
constexpr int64_t kFull = 256 * 16;      // wavefronts below which a row is spread over more lanes
constexpr int64_t kMostRows = INT64_C(1) << 40;
constexpr int kMostClasses = 1 << kIndexBits;
constexpr int64_t kFillParts = 512;      // workgroups that few long rows are cut into, at least
constexpr int64_t kPartVectors = 512;    // vectors of such a part, at least (rows of fewer than eight such parts are left whole: a join takes 4 us)
constexpr int kLongestRow = 1024 * 32;   // elements that a workgroup holds

template <typename T>
constexpr int kVec = 16 / sizeof(T);

int64_t row_parts(int64_t N, int64_t C, int vec)
{
    const int64_t nvec = (C + vec - 1) / vec, parts = (C + kLongestRow - 1) / kLongestRow;
    if (N * parts >= kFillParts || nvec < 8 * kPartVectors) return parts;
    return std::max(parts, std::min(nvec / kPartVectors, (kFillParts + N - 1) / N));
}

// Lanes of a row's team: `least`, or as few as hold it in `most` vectors each; more, up to `widest`, where the rows make too few wavefronts.  Answers go by 32
// elements a lane (us, 32 / 16: 500,000 x 47 in bf16, eight best 31 / 43; 200,000 x 172, five best 38 / 47), sorted lists of more than eight places by 16, for
// the registers; distillation by 4 vectors (100,000 x 300, 32 entries: 8 vectors 68, 4 vectors 63).
int team_lanes(int64_t N, int64_t nvec, int least, int most, int widest = 32)
{
    int lanes = least;
    while (lanes < widest && nvec > lanes * most) lanes *= 2;
    while (lanes < widest && nvec > lanes && N * lanes / 64 < kFull) lanes *= 2;
    return lanes;
}

template <typename T, int VEC, int NV, int TPR, int KT>
gp_status launch_short(const AnswerArgs& a, hipStream_t stream)
{
    constexpr int TEAMS = 256 / TPR;
    profile_begin("gp_answer_short", stream);
    hipLaunchKernelGGL((gp_answer_short<T, VEC, NV, TPR, KT>), dim3((unsigned)std::min((a.N + TEAMS - 1) / TEAMS, kMaxBlocks)), dim3(256), 0, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    return GP_OK;
}
// Elements of a row that lists of more than 8 places are kept in registers for; beyond, a wavefront's bound finds them.  us, bound / list in bf16: 246,153 x 260, 20 places
// 289 / 326, 130,000 x 500, 32 places 163 / 177, 3,000 x 300, 20 places 8.0 / 9.6.  A list would be sooner for 9 to 16 places there (12 places 241 / 198, 129 / 109) and
// for 33 to 64 up to 256 elements (320,000 x 200, 64 places 573 / 324; in fp32 378 / 322): those limits are too low.
constexpr int kListRow = 256, kLongListRow = 128;

template <typename T, int VEC, int NV, int TPR>
gp_status launch_short(const AnswerArgs& a, hipStream_t stream)
{
    const int places = std::min(a.k, a.C);
    if (places == 0) return launch_short<T, VEC, NV, TPR, 0>(a, stream);
    if (places == 1) return launch_short<T, VEC, NV, TPR, 1>(a, stream);
    if (places <= 4) return launch_short<T, VEC, NV, TPR, 4>(a, stream);
    if (places <= 8) return launch_short<T, VEC, NV, TPR, 8>(a, stream);
    if constexpr (NV * VEC <= 16 && VEC > 1) {
        if constexpr (TPR * 16 <= kListRow) {
            if (places <= 16) return launch_short<T, VEC, NV, TPR, 16>(a, stream);
            if (places <= 32) return launch_short<T, VEC, NV, TPR, 32>(a, stream);
        }
        if constexpr (TPR * 16 <= kLongListRow) return launch_short<T, VEC, NV, TPR, 64>(a, stream);
    }
    return fail(GP_ERR_UNSUPPORTED, "no kernel for %d alternatives of %d classes", a.k, a.C);
}
template <typename T, int VEC, int TPR>
gp_status launch_short(const AnswerArgs& a, hipStream_t stream)
{
    const int need = (a.nvec + TPR - 1) / TPR;
    if (need == 1) return launch_short<T, VEC, 1, TPR>(a, stream);
    if (need == 2) return launch_short<T, VEC, 2, TPR>(a, stream);
    if (need == 3) return launch_short<T, VEC, 3, TPR>(a, stream);
    if (need == 4) return launch_short<T, VEC, 4, TPR>(a, stream);
    if constexpr (VEC < 8) return need <= 6 ? launch_short<T, VEC, 6, TPR>(a, stream) : launch_short<T, VEC, 8, TPR>(a, stream);
    return fail(GP_ERR_UNSUPPORTED, "no kernel for %d classes", a.C);
}
// Vectors of a row that a wavefront takes by itself: without barriers it is done sooner than a workgroup, where there are rows enough (us, a wavefront / 256 lanes:
// 58,181 x 1100 in fp32, five best 86 / 160, loss and gradient 107 / 164; 25,000 x 2500 in bf16 59 / 82, 16,000 x 4000 38 / 53, 500 x 4000 8.7 / 6.2).
int64_t one_wavefront(int64_t items) { return items >= 2048 ? 512 : 256; }

template <typename T, int VEC, int NV, int TPR>
gp_status launch_rows(const AnswerArgs& a, hipStream_t stream)
{
    constexpr int BLOCK = TPR < 256 ? 256 : TPR, TEAMS = BLOCK / TPR;
    const int64_t items = a.N * a.parts;
    profile_begin("gp_answer_rows", stream);
    hipLaunchKernelGGL((gp_answer_rows<T, VEC, NV, TPR>), dim3((unsigned)std::min((items + TEAMS - 1) / TEAMS, kMaxBlocks)), dim3(BLOCK), 0, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    return GP_OK;
}
template <typename T, int VEC, int TPR>
gp_status launch_rows(const AnswerArgs& a, int64_t longest, hipStream_t stream)
{
    if (longest <= TPR) return launch_rows<T, VEC, 1, TPR>(a, stream);
    if (longest <= 2 * TPR) return launch_rows<T, VEC, 2, TPR>(a, stream);
    if (longest <= 4 * TPR) return launch_rows<T, VEC, 4, TPR>(a, stream);
    return launch_rows<T, VEC, 8, TPR>(a, stream);
}
// Rows of a wavefront or more, or parts of them (us, 256 lanes / 512: 7,111 x 9000 in bf16, five best 51 / 62; 12,800 x 5000 in fp32 67 / 91)
template <typename T>
gp_status launch_rows(const AnswerArgs& a, hipStream_t stream)
{
    const int64_t longest = (a.nvec + a.parts - 1) / a.parts;
    if (longest <= one_wavefront(a.N * a.parts)) return launch_rows<T, kVec<T>, 64>(a, longest, stream);
    if (longest <= 2048) return launch_rows<T, kVec<T>, 256>(a, longest, stream);
    if (longest <= 4096) return launch_rows<T, kVec<T>, 512>(a, longest, stream);
    if constexpr (kLongestRow > 4096 * kVec<T>)  // (a part is of kLongestRow elements at most: in bf16 none comes here)
        return launch_rows<T, kVec<T>, 1024>(a, longest, stream);
    return fail(GP_ERR_UNSUPPORTED, "no kernel for %lld vectors in one part", (long long)longest);
}

template <typename T>
gp_status launch_answer(AnswerArgs a, char* workspace, hipStream_t stream)
{
    constexpr int VEC = kVec<T>;
    if (a.C < VEC) {  // (a lane to a row)
        a.nvec = a.C;
        return launch_short<T, 1, 1>(a, stream);
    }
    a.nvec = (a.C + VEC - 1) / VEC;
    const int places = std::min(a.k, a.C);
    if (places <= 8 ? a.nvec <= 128 : a.C <= (places <= 32 ? kListRow : kLongListRow)) {
        switch (team_lanes(a.N, a.nvec, 2, (places <= 8 ? 32 : 16) / VEC, places <= 8 ? 32 : (places <= 32 ? kListRow : kLongListRow) / 16)) {
        case 2: return launch_short<T, VEC, 2>(a, stream);
        case 4: return launch_short<T, VEC, 4>(a, stream);
        case 8: return launch_short<T, VEC, 8>(a, stream);
        case 16: return launch_short<T, VEC, 16>(a, stream);
        default: return launch_short<T, VEC, 32>(a, stream);
        }
    }
    a.parts = (int)row_parts(a.N, a.C, VEC);
    a.partial = (float*)workspace;
    a.keys = (uint64_t*)(workspace + 16 * a.N * a.parts);
    gp_status st = launch_rows<T>(a, stream);
    if (st != GP_OK || a.parts == 1) return st;
    profile_begin("gp_answer_join", stream);
    const dim3 grid((unsigned)std::min(a.N, kMaxBlocks));
    if ((int64_t)a.parts * std::max(a.k, 1) <= 256)
        hipLaunchKernelGGL((gp_answer_join<T, 64>), grid, dim3(64), 0, stream, a);
    else
        hipLaunchKernelGGL((gp_answer_join<T, 1024>), grid, dim3(1024), 0, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    return GP_OK;
}

template <typename T, int VEC, int NV, int TPR, int PER>
gp_status launch_distill_short(const DistillArgs& a, hipStream_t stream)
{
    constexpr int TEAMS = 256 / TPR;
    profile_begin("gp_distill_short", stream);
    hipLaunchKernelGGL((gp_distill_short<T, VEC, NV, TPR, PER>), dim3((unsigned)std::min((a.N + TEAMS - 1) / TEAMS, kMaxBlocks)), dim3(256), 0, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    return GP_OK;
}
template <typename T, int VEC, int NV, int TPR>
gp_status launch_distill_short(const DistillArgs& a, hipStream_t stream)
{
    if (a.K <= TPR) return launch_distill_short<T, VEC, NV, TPR, 1>(a, stream);
    if (a.K <= 2 * TPR) return launch_distill_short<T, VEC, NV, TPR, 2>(a, stream);
    if constexpr (TPR <= 16)
        if (a.K <= 4 * TPR) return launch_distill_short<T, VEC, NV, TPR, 4>(a, stream);
    if constexpr (TPR <= 8)
        if (a.K <= 8 * TPR) return launch_distill_short<T, VEC, NV, TPR, 8>(a, stream);
    return fail(GP_ERR_UNSUPPORTED, "no kernel for %d entries of %d classes", a.K, a.C);
}
template <typename T, int VEC, int TPR>
gp_status launch_distill_short(const DistillArgs& a, hipStream_t stream)
{
    const int need = (a.nvec + TPR - 1) / TPR;
    if (need == 1) return launch_distill_short<T, VEC, 1, TPR>(a, stream);
    if (need == 2) return launch_distill_short<T, VEC, 2, TPR>(a, stream);
    if (need == 3) return launch_distill_short<T, VEC, 3, TPR>(a, stream);
    if constexpr (VEC == 1)
        if (need > 4) return need <= 6 ? launch_distill_short<T, VEC, 6, TPR>(a, stream) : launch_distill_short<T, VEC, 8, TPR>(a, stream);
    return launch_distill_short<T, VEC, 4, TPR>(a, stream);
}
template <typename T, int VEC, int NV, int TPR>
gp_status launch_distill_rows(const DistillArgs& a, hipStream_t stream)
{
    constexpr int BLOCK = TPR < 256 ? 256 : TPR, TEAMS = BLOCK / TPR;
    const int64_t items = a.N * a.parts;
    profile_begin("gp_distill_rows", stream);
    hipLaunchKernelGGL((gp_distill_rows<T, VEC, NV, TPR>), dim3((unsigned)std::min((items + TEAMS - 1) / TEAMS, kMaxBlocks)), dim3(BLOCK), 0, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    return GP_OK;
}
template <typename T, int VEC, int TPR>
gp_status launch_distill_rows(const DistillArgs& a, int64_t longest, hipStream_t stream)
{
    if (longest <= TPR) return launch_distill_rows<T, VEC, 1, TPR>(a, stream);
    if (longest <= 2 * TPR) return launch_distill_rows<T, VEC, 2, TPR>(a, stream);
    if (longest <= 4 * TPR) return launch_distill_rows<T, VEC, 4, TPR>(a, stream);
    return launch_distill_rows<T, VEC, 8, TPR>(a, stream);
}
template <typename T>
gp_status launch_distill_rows(const DistillArgs& a, hipStream_t stream)
{
    const int64_t longest = (a.nvec + a.parts - 1) / a.parts;
    if (longest <= one_wavefront(a.N * a.parts)) return launch_distill_rows<T, kVec<T>, 64>(a, longest, stream);
    if (longest <= 2048) return launch_distill_rows<T, kVec<T>, 256>(a, longest, stream);
    if (longest <= 4096) return launch_distill_rows<T, kVec<T>, 512>(a, longest, stream);
    return launch_distill_rows<T, kVec<T>, 1024>(a, longest, stream);
}

template <typename T>
gp_status launch_distill(DistillArgs a, char* workspace, hipStream_t stream)
{
    constexpr int VEC = kVec<T>;
    a.parts = 1;
    if (a.C < VEC) {
        a.nvec = a.C;
        return a.K <= 8 ? launch_distill_short<T, 1, 1>(a, stream) : launch_distill_short<T, 1, 1, 8>(a, stream);
    }
    a.nvec = (a.C + VEC - 1) / VEC;
    if (a.nvec <= 128) {
        switch (team_lanes(a.N, a.nvec, a.K > 32 ? 8 : a.K > 16 || a.nvec > 4 ? 4 : 2, 4)) {  // (at most eight entries to a lane)
        case 2: return launch_distill_short<T, VEC, 2>(a, stream);
        case 4: return launch_distill_short<T, VEC, 4>(a, stream);
        case 8: return launch_distill_short<T, VEC, 8>(a, stream);
        case 16: return launch_distill_short<T, VEC, 16>(a, stream);
        default: return launch_distill_short<T, VEC, 32>(a, stream);
        }
    }
    a.parts = (int)row_parts(a.N, a.C, VEC);
    // a gradient of rows in parts reads them twice: in bf16 up to 65,536 classes are held by one workgroup where there are rows enough for all units, though
    // it has one to itself then (1,939 x 33,000 105 -> 87 us, 1,280 x 50,000 88 -> 72; without a gradient it would lose)
    if (a.grad && !a.from && a.N >= 256 && a.C <= 1024 * 8 * VEC) a.parts = 1;
    if (a.parts == 1 || a.from) return launch_distill_rows<T>(a, stream);
    AnswerArgs s{};
    s.x = a.x, s.ld = a.ld, s.N = a.N, s.C = a.C, s.nvec = a.nvec, s.scale = 1.0f / a.T, s.parts = a.parts;
    s.partial = a.partial = (float*)workspace;
    gp_status st = launch_rows<T>(s, stream);
    if (st != GP_OK) return st;
    if (!a.stats) a.stats = (float*)(workspace + 16 * a.N * a.parts);
    profile_begin("gp_distill_join", stream);
    hipLaunchKernelGGL(gp_distill_join<T>, dim3((unsigned)std::min((a.N + 3) / 4, kMaxBlocks)), dim3(256), 0, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    if (!a.grad) return GP_OK;
    a.from = a.stats;
    return launch_distill_rows<T>(a, stream);
}

template <typename T, int VEC>
gp_status launch_answer_grad(AnswerGradArgs a, hipStream_t stream)
{
    a.nvec = (a.C + VEC - 1) / VEC;
    const int64_t blocks = (a.N * a.nvec + 511) / 512;
    profile_begin("gp_answer_grad", stream);
    hipLaunchKernelGGL((gp_answer_grad<T, VEC>), dim3((unsigned)std::min(blocks, kMaxBlocks)), dim3(256), 0, stream, a);
    profile_end(stream);
    GP_HIP(hipGetLastError());
    return GP_OK;
}
template <typename T>
gp_status launch_answer_grad(const AnswerGradArgs& a, hipStream_t stream)
{
    return a.C >= kVec<T> ? launch_answer_grad<T, kVec<T>>(a, stream) : launch_answer_grad<T, 1>(a, stream);
}

// Bytes of the parts' results, whichever type the logits are of.
int64_t parts_bytes(int64_t N, int32_t C, int32_t k)
{
    if (N == 0) return 0;
    int64_t most = 0;
    for (int vec : {kVec<float>, kVec<bf16_t>}) {
        const int64_t parts = row_parts(N, C, vec);
        if (parts > 1) most = std::max(most, N * parts * (16 + 8 * (int64_t)k));
    }
    return (most + 255) / 256 * 256;
}

bool known(gp_dtype t) { return t == GP_F32 || t == GP_BF16; }

// What every call asks of the logits; `done` where there are none.
gp_status check_logits(int64_t ld, gp_dtype dtype, int64_t N, int32_t C)
{
    if (!known(dtype)) return fail(GP_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
    if (N < 0 || C < 1 || ld < C) return fail(GP_ERR_INVALID_ARG, "need N >= 0, C >= 1, ld >= C");
    if (N > kMostRows || C > kMostClasses) return fail(GP_ERR_UNSUPPORTED, "more than 2^40 rows or 2^28 classes");
    return GP_OK;
}
gp_status check_workspace(const void* workspace, int64_t bytes, int64_t need)
{
    if (need > 0 && (!workspace || bytes < need || (uintptr_t)workspace % 256 != 0))
        return fail(GP_ERR_INVALID_ARG, "need a workspace of %lld bytes on a 256-byte boundary", (long long)need);
    return GP_OK;
}
bool good_scale(float s) { return s > 0.0f && s <= 1e30f && s >= 1e-30f; }

gp_status log_probs(const void* x, int64_t ld, gp_dtype dtype, int64_t N, int32_t C, const void* tokens, gp_index index, float scale, float* logp, float* entropy,
                    int32_t k, int32_t* top_index, float* top_logp, float* stats, void* workspace, int64_t bytes, hipStream_t stream)
{
    gp_status st = check_logits(ld, dtype, N, C);
    if (st != GP_OK) return st;
    if (index != GP_I32 && index != GP_I64) return fail(GP_ERR_INVALID_ARG, "unknown index type %d", (int)index);
    if (!good_scale(scale)) return fail(GP_ERR_INVALID_ARG, "need a scale within 1e-30 .. 1e30");
    if (k < 0) return fail(GP_ERR_INVALID_ARG, "need k >= 0");
    if (k > kMostTop) return fail(GP_ERR_UNSUPPORTED, "more than %d alternatives", kMostTop);
    if (N == 0) return GP_OK;
    if (!x || (logp && !tokens) || (k > 0 && (!top_index || !top_logp))) return fail(GP_ERR_INVALID_ARG, "NULL argument");
    if ((st = check_workspace(workspace, bytes, parts_bytes(N, C, k))) != GP_OK) return st;
    if (!logp && !entropy && k == 0 && !stats) return GP_OK;
    AnswerArgs a{};
    a.x = x, a.ld = ld, a.N = N, a.C = C, a.tokens = tokens, a.wide = index == GP_I64, a.scale = scale, a.logp = logp, a.entropy = entropy, a.stats = stats,
    a.k = k, a.top_index = top_index, a.top_logp = top_logp, a.parts = 1;
    return dtype == GP_F32 ? launch_answer<float>(a, (char*)workspace, stream) : launch_answer<bf16_t>(a, (char*)workspace, stream);
}

gp_status log_probs_grad(const void* x, int64_t ld, gp_dtype dtype, int64_t N, int32_t C, const void* tokens, gp_index index, float scale, const float* stats,
                         const float* entropy, const float* g1, int64_t s1, const float* g2, int64_t s2, void* grad, int64_t ldg, hipStream_t stream)
{
    gp_status st = check_logits(ld, dtype, N, C);
    if (st != GP_OK) return st;
    if (index != GP_I32 && index != GP_I64) return fail(GP_ERR_INVALID_ARG, "unknown index type %d", (int)index);
    if (!good_scale(scale)) return fail(GP_ERR_INVALID_ARG, "need a scale within 1e-30 .. 1e30");
    if (ldg < C || (s1 != 0 && s1 != 1) || (s2 != 0 && s2 != 1)) return fail(GP_ERR_INVALID_ARG, "need ldg >= C, distances of 0 or 1");
    if (N == 0) return GP_OK;
    if (!x || !stats || !grad || (g1 && !tokens) || (g2 && !entropy)) return fail(GP_ERR_INVALID_ARG, "NULL argument");
    if (N > (INT64_C(1) << 62) / C) return fail(GP_ERR_OVERFLOW, "N x C does not fit 62 bits");
    AnswerGradArgs a{};
    a.x = x, a.ld = ld, a.N = N, a.C = C, a.tokens = tokens, a.wide = index == GP_I64, a.scale = scale, a.stats = stats, a.entropy = entropy, a.g1 = g1, a.s1 = s1,
    a.g2 = g2, a.s2 = s2, a.grad = grad, a.ldg = ldg;
    return dtype == GP_F32 ? launch_answer_grad<float>(a, stream) : launch_answer_grad<bf16_t>(a, stream);
}

int64_t distill_bytes(int64_t N, int32_t C)
{
    const int64_t parts = parts_bytes(N, C, 0);
    return parts ? parts + (8 * N + 255) / 256 * 256 : 0;
}

gp_status distill(const void* x, int64_t ld, gp_dtype dtype, int64_t N, int32_t C, const void* index, int64_t ldi, gp_index index_type, const void* teacher,
                  int64_t ldt, gp_dtype teacher_dtype, int32_t K, float T, float* loss, float* stats, const float* from, const float* g, int64_t sg, void* grad,
                  int64_t ldg, void* workspace, int64_t bytes, hipStream_t stream)
{
    gp_status st = check_logits(ld, dtype, N, C);
    if (st != GP_OK) return st;
    if (index_type != GP_I32 && index_type != GP_I64) return fail(GP_ERR_INVALID_ARG, "unknown index type %d", (int)index_type);
    if (!known(teacher_dtype)) return fail(GP_ERR_INVALID_ARG, "unknown dtype %d", (int)teacher_dtype);
    if (K < 1 || ldi < K || ldt < K) return fail(GP_ERR_INVALID_ARG, "need K >= 1, ldi >= K, ldt >= K");
    if (K > kMostTop) return fail(GP_ERR_UNSUPPORTED, "more than %d entries", kMostTop);
    if (!(T >= 1e-15f && T <= 1e15f)) return fail(GP_ERR_INVALID_ARG, "need a temperature within 1e-15 .. 1e15");  // (its square is a number too)
    if (grad && (ldg < C || (sg != 0 && sg != 1))) return fail(GP_ERR_INVALID_ARG, "need ldg >= C, a distance of 0 or 1");
    if (N == 0) return GP_OK;
    if (!x || !index || !teacher || (grad && !g)) return fail(GP_ERR_INVALID_ARG, "NULL argument");
    if (!from && (st = check_workspace(workspace, bytes, distill_bytes(N, C))) != GP_OK) return st;
    if (!loss && !stats && !grad) return GP_OK;
    DistillArgs a{};
    a.x = x, a.ld = ld, a.N = N, a.C = C, a.index = index, a.wide = index_type == GP_I64, a.ldi = ldi, a.teacher = teacher, a.ldv = ldt,
    a.wide_teacher = teacher_dtype == GP_F32, a.K = K, a.T = T, a.loss = loss, a.stats = stats, a.from = from, a.g = g, a.sg = sg, a.grad = grad, a.ldg = ldg;
    return dtype == GP_F32 ? launch_distill<float>(a, (char*)workspace, stream) : launch_distill<bf16_t>(a, (char*)workspace, stream);
}

}  // namespace

}  // namespace gp

extern "C" int64_t gp_log_probs_workspace(int64_t N, int32_t C, int32_t k)
{
    if (N < 0 || N > gp::kMostRows || C < 1 || C > gp::kMostClasses || k < 0 || k > gp::kMostTop) return -1;
    return gp::parts_bytes(N, C, k);
}

extern "C" gp_status gp_log_probs(const void* logits, int64_t ld, gp_dtype dtype, int64_t N, int32_t C, const void* tokens, gp_index index, float scale, float* logp,
                                  float* entropy, int32_t k, int32_t* top_index, float* top_logp, float* stats, void* workspace, int64_t workspace_bytes,
                                  void* hip_stream)
{
    try {
        return gp::log_probs(logits, ld, dtype, N, C, tokens, index, scale, logp, entropy, k, top_index, top_logp, stats, workspace, workspace_bytes,
                             (hipStream_t)hip_stream);
    } catch (const std::exception& e) {
        return gp::fail(GP_ERR_OOM_HOST, "gp_log_probs: %s", e.what());
    }
}

extern "C" gp_status gp_log_probs_grad(const void* logits, int64_t ld, gp_dtype dtype, int64_t N, int32_t C, const void* tokens, gp_index index, float scale,
                                       const float* stats, const float* entropy, const float* grad_logp, int64_t stride_logp, const float* grad_entropy,
                                       int64_t stride_entropy, void* grad, int64_t ldg, void* hip_stream)
{
    try {
        return gp::log_probs_grad(logits, ld, dtype, N, C, tokens, index, scale, stats, entropy, grad_logp, stride_logp, grad_entropy, stride_entropy, grad, ldg,
                                  (hipStream_t)hip_stream);
    } catch (const std::exception& e) {
        return gp::fail(GP_ERR_OOM_HOST, "gp_log_probs_grad: %s", e.what());
    }
}

extern "C" int64_t gp_distill_workspace(int64_t N, int32_t C)
{
    if (N < 0 || N > gp::kMostRows || C < 1 || C > gp::kMostClasses) return -1;
    return gp::distill_bytes(N, C);
}

extern "C" gp_status gp_distill(const void* logits, int64_t ld, gp_dtype dtype, int64_t N, int32_t C, const void* teacher_index, int64_t ldi, gp_index index,
                                const void* teacher_logits, int64_t ldt, gp_dtype teacher_dtype, int32_t K, float temperature, float* loss, float* stats,
                                const float* grad_loss, int64_t stride_loss, void* grad, int64_t ldg, void* workspace, int64_t workspace_bytes, void* hip_stream)
{
    try {
        return gp::distill(logits, ld, dtype, N, C, teacher_index, ldi, index, teacher_logits, ldt, teacher_dtype, K, temperature, loss, stats, nullptr, grad_loss,
                           stride_loss, grad, ldg, workspace, workspace_bytes, (hipStream_t)hip_stream);
    } catch (const std::exception& e) {
        return gp::fail(GP_ERR_OOM_HOST, "gp_distill: %s", e.what());
    }
}

extern "C" gp_status gp_distill_grad(const void* logits, int64_t ld, gp_dtype dtype, int64_t N, int32_t C, const void* teacher_index, int64_t ldi, gp_index index,
                                     const void* teacher_logits, int64_t ldt, gp_dtype teacher_dtype, int32_t K, float temperature, const float* stats,
                                     const float* grad_loss, int64_t stride_loss, void* grad, int64_t ldg, void* hip_stream)
{
    try {
        if (N > 0 && (!stats || !grad)) return gp::fail(GP_ERR_INVALID_ARG, "NULL argument");
        return gp::distill(logits, ld, dtype, N, C, teacher_index, ldi, index, teacher_logits, ldt, teacher_dtype, K, temperature, nullptr, nullptr, stats, grad_loss,
                           stride_loss, grad, ldg, nullptr, 0, (hipStream_t)hip_stream);
    } catch (const std::exception& e) {
        return gp::fail(GP_ERR_OOM_HOST, "gp_distill_grad: %s", e.what());
    }
}
