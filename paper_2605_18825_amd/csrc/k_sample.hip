// Sampling a token per row of logits by temperature, top-k, top-p and min-p.
//
// Every part of the definition is a question to one order, by falling logit and rising index: the
// weight of its first k tokens, the shortest head that holds p of it, the token where u of it is
// passed.  So nothing is sorted but the few tokens that the answers lie among.  Weights
// exp((l - l_0) / T) are computed in 64 bits and held as whole multiples of 2^-43 (the sum of 2^20
// fits 64 bits): sums are exact, whatever their order, and LDS atomics can take them.
//
// A workgroup takes a row.  The first pass finds the maximum, and each thread keeps the maxima of 16
// groups of its logits: a later pass for the few largest logits reads those groups alone.
//   small k     the k-th largest of the threads' maxima bounds the k-th largest logit from below:
//               what is not below it is collected, a few more than k tokens.
//   otherwise   a second pass adds every token to a histogram over (l_0 - l) / T, 32 bins for a
//               factor of two: each bin's tokens and their weight.  The answers' bin follows, and
//               the tokens up to it are collected.
//   where these are many, only the tokens of the bins that the answers can lie in are: a bin is
//   2.2 % of weight wide, and what it leaves open of one answer leaves the next one a bin or two.
//   where these are more than LDS holds, each question is answered by itself: its bin, then
//   (a bin of many equal or near logits) 10 bits of the logit at a time, then the index.
//
// Bound by the logits' bytes with a small k: 256 rows of 131,072 bf16 logits 18.6 us, 3.6 TB/s with a
// few dependent steps behind it.  Otherwise by the histogram's pass, in vector instructions: for a row
// of 100,003 f32 logits it takes 57 thousand clocks, 26 thousand without the weights.  64 rows of 100,003 with
// nothing left out: 45 to 47 us by card; 700 rows of 50,001 with settings of their own: 72.5.
//
// Few rows of a large vocabulary leave most of the GPU idle: there the first two passes are launches
// of their own, a row's vectors over several workgroups, maxima and the histogram in the workspace (whole
// numbers added by atomics: in any order the same), and the rest is as above.
#include <algorithm>

#include "attn_tile.h"

namespace {

using attn::sum_upto;
using attn::uniform;
using attn::upto;

constexpr int LIST = 2048;           // tokens that are sorted in LDS
constexpr int PER_TWO = 32;          // bins of a factor of two in weight
constexpr int LIGHT = 47 * PER_TWO;  // the bin of tokens that weigh less than half a unit, as nothing
constexpr int BINS = 1536, DIGITS = 1024;
constexpr int GROUPS = 16;           // of a thread's logits
constexpr double ONE = 8796093022208.0;  // 2^43
constexpr float LOWEST = -__builtin_inff();
typedef attn::u64 u64;
static_assert(LIGHT < BINS, "");

struct Args {
    const void *logits;
    int64_t stride;
    const float *temperature, *top_p, *min_p, *u;
    const int32_t *top_k;
    int32_t *token, *kept;
    float *prob;
    int32_t vocab;
    char *work;
};

// A row's part of the workspace, where its passes are launches of their own.
constexpr int SPLIT_GROUPS = GROUPS * 1024, SPLIT_MAXES = 64;
struct Shelf {
    u64 mass[BINS];
    uint32_t count[BINS];
    float most[SPLIT_GROUPS];  // maxima of vectors i SPLIT_GROUPS + g, for each g
    float maxes[SPLIT_MAXES];  // the workgroups' maxima
};

// ------------------------------------------------------------- waves and workgroups
__device__ __forceinline__ uint32_t of_lane(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }
__device__ __forceinline__ u64 of_lane(u64 x, int lane) { return (u64)of_lane((uint32_t)(x >> 32), lane) << 32 | of_lane((uint32_t)x, lane); }
__device__ __forceinline__ float of_lane(float x, int lane) { return __uint_as_float(of_lane(__float_as_uint(x), lane)); }

struct Hist {
    u64 mass[BINS];
    uint32_t count[BINS];
};

struct Shared {
    Hist bins;
    union {  // (digits are done with when a list is summed)
        struct {
            u64 mass[DIGITS];
            uint32_t count[DIGITS];
        } digits;
        u64 sums[LIST];  // weights up to each token of the list, itself included
    };
    u64 list[LIST];  // key << 32 | index
    double power[PER_TWO];  // 2^(-j / 32) units
    u64 part[2][16];
    float edges[8];
    uint32_t n, found;
};

// f over the workgroup, in every thread; which: alternates between calls.
template <int NW, typename T, typename F>
__device__ __forceinline__ T over_all(Shared &s, int which, T x, T idle, F f)
{
    T *part = reinterpret_cast<T *>(s.part[which]);
    x = upto(x, idle, f);
    if (__lane_id() == SAE_WAVE - 1) part[threadIdx.x / SAE_WAVE] = x;
    __syncthreads();
    x = part[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) x = f(x, part[w]);
    return x;
}

// The sum over the threads before this one; which: alternates between calls.
template <int NW, typename T>
__device__ __forceinline__ T sum_before(Shared &s, int which, T x)
{
    T *part = reinterpret_cast<T *>(s.part[which]);
    const T mine = sum_upto(x);
    if (__lane_id() == SAE_WAVE - 1) part[threadIdx.x / SAE_WAVE] = mine;
    __syncthreads();
    T before = mine - x;
#pragma unroll
    for (int w = 0; w < NW - 1; ++w)
        if (w < (int)threadIdx.x / SAE_WAVE) before += part[w];
    return before;
}

// ------------------------------------------------------------- a row
// Ascending whole numbers for falling logits.
__device__ __forceinline__ uint32_t key_of(float l)
{
    const uint32_t b = __float_as_uint(l + 0.0f);  // (-0 and 0 are equal)
    return b >> 31 ? b : ~b & 0x7FFFFFFFu;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key >> 31 ? key : ~key & 0x7FFFFFFFu); }

template <int DT, int THREADS>
struct Row {
    static constexpr int E = DT == SAE_ROWS_F32 ? 4 : 8;  // logits of 16 bytes
    static constexpr int SIZE = 16 / E, UN = 4;
    const char *at, *body;
    int n, head, vectors;  // logits before the first 16-byte boundary, whole vectors behind them
    bool infinite;         // +inf is the largest: it counts as 0 then, and other logits as -2^127
    float most[GROUPS];    // maxima of the thread's groups: group g has vectors (16 i + g) THREADS + thread
    float edge;            // the thread's logit before or behind the vectors, and its index
    int edge_at;

    __device__ __forceinline__ Row(const void *p, int vocab) : at(static_cast<const char *>(p)), n(vocab), infinite(false)
    {
        head = min((int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / SIZE, n);
        vectors = (n - head) / E;
        body = at + head * SIZE;
        const int t = threadIdx.x, tail = n - head - vectors * E;  // both below E
        edge_at = t < head ? t : t >= SAE_WAVE && t < SAE_WAVE + tail ? n - tail + t - SAE_WAVE : -1;
    }
    __device__ __forceinline__ float mapped(float l) const
    {
        return infinite ? (l == __builtin_inff() ? 0.0f : l > LOWEST ? -0x1p127f : LOWEST) : l;
    }
    static __device__ __forceinline__ float wide(u32x4 x, int i)
    {
        if constexpr (DT == SAE_ROWS_F32) return __uint_as_float(x[i]);
        else return i & 1 ? attn::high<DT == SAE_KV_F16>(x[i / 2]) : attn::low<DT == SAE_KV_F16>(x[i / 2]);
    }
    __device__ __forceinline__ u32x4 vector(int v) const { return *reinterpret_cast<const u32x4 *>(body + (int64_t)v * 16); }

    __device__ __forceinline__ void load_edge()
    {
        edge = LOWEST;
        if (edge_at >= 0) {
            if constexpr (DT == SAE_ROWS_F32) edge = fmaxf(reinterpret_cast<const float *>(at)[edge_at], LOWEST);
            else edge = fmaxf(attn::low<DT == SAE_KV_F16>((uint32_t)reinterpret_cast<const uint16_t *>(at)[edge_at]), LOWEST);
        }
    }
    // The maxima that the first launch has left; returns the thread's largest.
    __device__ __forceinline__ float maxima_of(const Shelf &shelf)
    {
        static_assert(GROUPS * THREADS == SPLIT_GROUPS || THREADS != 1024, "a thread has groups t, t + THREADS, ...");
        load_edge();
        float m = edge;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const int v = g * THREADS + (int)threadIdx.x;
            most[g] = v < vectors ? shelf.most[v] : LOWEST;
            m = fmaxf(m, most[g]);
        }
        return m;
    }
    // The first pass: the thread's maxima; returns the largest.
    __device__ __forceinline__ float maxima()
    {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) most[g] = LOWEST;
        load_edge();
#pragma unroll 1
        for (int v0 = 0; v0 < vectors; v0 += GROUPS * THREADS) {
#pragma unroll
            for (int g0 = 0; g0 < GROUPS; g0 += UN) {
                if (v0 + g0 * THREADS >= vectors) break;  // uniform
                u32x4 x[UN];
#pragma unroll
                for (int i = 0; i < UN; ++i) x[i] = vector(min(v0 + (g0 + i) * THREADS + (int)threadIdx.x, vectors - 1));
#pragma unroll
                for (int i = 0; i < UN; ++i) {
                    float m = most[g0 + i];
#pragma unroll
                    for (int e = 0; e < E; ++e) m = fmaxf(m, wide(x[i], e));
                    most[g0 + i] = v0 + (g0 + i) * THREADS + (int)threadIdx.x < vectors ? m : most[g0 + i];
                }
            }
        }
        float m = edge;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) m = fmaxf(m, most[g]);
        return m;
    }
    // What the maxima and the edge are where +inf is the largest logit.
    __device__ __forceinline__ void set_infinite()
    {
        infinite = true;
        edge = mapped(edge);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) most[g] = mapped(most[g]);
    }
    // f(logit, index) for every logit.
    template <typename F>
    __device__ __forceinline__ void each(F f) const
    {
        each(LOWEST, f, [](float) {});
    }
    // f(logit, index) for every logit; low(logit) for those of vectors that lie below `bound` whole.
    template <typename F, typename L>
    __device__ __forceinline__ void each(float bound, F f, L low) const
    {
        each_of(0, vectors, bound, f, low);
        if (edge_at >= 0) f(edge, edge_at);
    }
    // The same for vectors first .. last - 1.
    template <typename F, typename L>
    __device__ __forceinline__ void each_of(int first, int last, float bound, F f, L low) const
    {
#pragma unroll 1
        for (int v = first + (int)threadIdx.x; v < last; v += THREADS * UN) {
            u32x4 x[UN];
#pragma unroll
            for (int k = 0; k < UN; ++k) x[k] = vector(min(v + k * THREADS, last - 1));
#pragma unroll
            for (int k = 0; k < UN; ++k)
                if (v + k * THREADS < last) {
                    if (bound > LOWEST && !infinite) {  // uniform
                        float m = wide(x[k], 0);
#pragma unroll
                        for (int i = 1; i < E; ++i) m = fmaxf(m, wide(x[k], i));
                        if (!(m >= bound)) {
#pragma unroll
                            for (int i = 0; i < E; ++i) low(wide(x[k], i));
                            continue;
                        }
                    }
                    use(x[k], v + k * THREADS, f);
                }
        }
    }
    // Appends the indexes of all logits with pred(logit) to `list`, at most `room`; n: counts them (all).
    // Bits for four vectors at a time: a test has no branch, and a thread with any takes one place for all of them.
    template <typename P>
    __device__ __forceinline__ void collect(uint32_t *list, uint32_t *n, int room, P pred) const
    {
        auto put = [&](uint32_t at, int i) {
            if (at < (uint32_t)room) list[at] = (uint32_t)i;
        };
        if (infinite) {  // uniform
            each([&](float l, int i) {
                if (pred(l)) put(atomicAdd(n, 1u), i);
            });
            return;
        }
#pragma unroll 1
        for (int v = threadIdx.x; v < vectors; v += THREADS * UN) {
            u32x4 x[UN];
#pragma unroll
            for (int k = 0; k < UN; ++k) x[k] = vector(min(v + k * THREADS, vectors - 1));
            uint32_t bits = 0;
#pragma unroll
            for (int k = 0; k < UN; ++k)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    bits |= pred(wide(x[k], i)) ? 1u << (k * E + i) : 0u;
                }
            const int there = min((vectors - v + THREADS - 1) / THREADS, UN) * E;  // bits of vectors that there are
            bits &= (uint32_t)((1ull << there) - 1);
            if (!bits) continue;
            uint32_t at = atomicAdd(n, (uint32_t)__builtin_popcount(bits));
            while (bits) {
                const int b = __builtin_ctz(bits);
                bits &= bits - 1;
                put(at++, head + (v + b / E * THREADS) * E + b % E);
            }
        }
        if (edge_at >= 0 && pred(edge)) put(atomicAdd(n, 1u), edge_at);
    }
    // The logit at an index.
    __device__ __forceinline__ float logit(int i) const
    {
        if constexpr (DT == SAE_ROWS_F32) return mapped(reinterpret_cast<const float *>(at)[i]);
        else return mapped(attn::low<DT == SAE_KV_F16>((uint32_t)reinterpret_cast<const uint16_t *>(at)[i]));
    }
    // The bound where a whole wave's vectors of some group lie below it, else -inf: with a few below it among
    // others a wave goes both ways.
    __device__ __forceinline__ float any_below(float bound) const
    {
        bool found = false;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) found |= __all(most[g] < bound) && g * THREADS < vectors;
        return found ? bound : LOWEST;
    }
    // f(logit, index) for every logit >= bound, and others.
    template <typename F>
    __device__ __forceinline__ void some(float bound, F f) const
    {
        uint32_t groups = 0;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) groups |= most[g] >= bound ? 1u << g : 0u;
        while (groups) {
            const int g = __builtin_ctz(groups);
            groups &= groups - 1;
#pragma unroll 1
            for (int v = g * THREADS + (int)threadIdx.x; v < vectors; v += GROUPS * THREADS) use(vector(v), v, f);
        }
        if (edge >= bound && edge_at >= 0) f(edge, edge_at);
    }

private:
    template <typename F>
    __device__ __forceinline__ void use(u32x4 x, int v, F f) const
    {
        if (infinite) {  // uniform
#pragma unroll 1
            for (int i = 0; i < E; ++i) f(mapped(wide(x, i)), head + v * E + i);
            return;
        }
#pragma unroll
        for (int i = 0; i < E; ++i) f(wide(x, i), head + v * E + i);
    }
};

// A row's weights and bins.
struct Scale {
    double top, c;        // l_0; 32 log2 e / T
    const double *power;

    // (l_0 - l) / T in 32nds of a factor of two, as a whole number and a rest in +-1/2; NaN and -inf: LIGHT
    __device__ __forceinline__ int split(float l, double &rest) const
    {
        const double y = __builtin_fmin((top - (double)l) * c, (double)LIGHT);
        const double t = y + 4503599627370496.0;  // 2^52: the sum's last bits are y's whole number
        rest = y - (t - 4503599627370496.0);
        return (int)__double2loint(t);
    }
    __device__ __forceinline__ int bin(float l) const
    {
        double rest;
        return split(l, rest);
    }
    // exp((l - l_0) / T) in units of 2^-43 by the rest's Taylor series (next term 2e-15) and a table of 32 powers.
    __device__ __forceinline__ u64 weight(int n, double rest) const
    {
        constexpr double A = -0.693147180559945309417 / PER_TWO;
        double y = __builtin_fma(rest, A * A * A * A * A / 120, A * A * A * A / 24);
        y = __builtin_fma(rest, y, A * A * A / 6);
        y = __builtin_fma(rest, y, A * A / 2);
        y = __builtin_fma(rest, y, A);
        y = __builtin_fma(rest, y, 1.0);
        // 2^(-n / 32): the table's by the last bits of n, the others are the exponent's
        const double p = power[n & (PER_TWO - 1)];
        const double q = __hiloint2double(__double2hiint(p) - (int)((uint32_t)n / PER_TWO << 20), __double2loint(p));
        // rounded to a whole number by 2^52, whose last bit is 1
        return (u64)__double_as_longlong(__builtin_fma(y, q, 4503599627370496.0)) & 0xFFFFFFFFFFFFFull;
    }
    __device__ __forceinline__ u64 weight(float l) const
    {
        double rest;
        const int n = split(l, rest);
        return weight(n, rest);
    }
    // A logit that those of bins 0 .. b are not below, and bins from b + 2 on are not above.
    __device__ __forceinline__ float floor_of(int b) const { return __double2float_rd(top - (b + 1.0) / c); }
};

// The lowest logit of bins 0 .. b (b < LIGHT), by a wave: bins do not fall as keys rise.
__device__ __forceinline__ float lowest_of(const Scale &sc, int b)
{
    constexpr uint32_t FIRST = 0x00800000u, LAST = 0xFF7FFFFFu;  // keys of the largest and the lowest float
    auto inside = [&](uint32_t k) {
        const float l = logit_of(k);
        return (double)l >= sc.top || sc.bin(l) <= b;
    };
    {  // most often within a few floats of where the bin ends
        const uint32_t k = key_of((float)(sc.top - (b + 0.5) / sc.c)), from = k > FIRST + 32 && k < LAST - 64 ? k - 32 : FIRST;
        const u64 in = __ballot(inside(from + (uint32_t)__lane_id()));
        const int last = __builtin_popcountll(in) - 1;
        if (last >= 0 && last < SAE_WAVE - 1) return logit_of(from + last);
    }
    uint32_t lo = FIRST, n = LAST - FIRST + 1;  // the last key with a bin up to b lies in [lo, lo + n)
    while (n > 1) {
        const uint32_t step = (n + SAE_WAVE - 1) / SAE_WAVE, k = (uint32_t)__lane_id() * step;
        const u64 in = __ballot(k < n && inside(lo + min(k, n - 1)));
        const uint32_t skip = in ? (uint32_t)(63 - __builtin_clzll(in)) * step : 0;
        lo += skip;
        n = min(step, n - skip);
    }
    return logit_of(lo);
}

// Counts and masses up to each bin, itself included.
template <int NW, int N>
__device__ __forceinline__ void accumulate(Shared &s, u64 *mass, uint32_t *count)
{
    constexpr int PER = (N + NW * SAE_WAVE - 1) / (NW * SAE_WAVE);
    const int i0 = threadIdx.x * PER;
    u64 m[PER];
    uint32_t c[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        m[i] = i0 + i < N ? mass[i0 + i] : 0;
        c[i] = i0 + i < N ? count[i0 + i] : 0;
        if (i) {
            m[i] += m[i - 1];
            c[i] += c[i - 1];
        }
    }
    const uint32_t cb = sum_before<NW>(s, 0, c[PER - 1]);
    const u64 mb = sum_before<NW>(s, 1, m[PER - 1]);
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (i0 + i < N) {
            mass[i0 + i] = mb + m[i];
            count[i0 + i] = cb + c[i];
        }
    __syncthreads();
}

// The first i < n <= 4096 for which pred(i) holds (it holds from there on); n - 1 where none does.  Every wave by itself.
template <typename P>
__device__ __forceinline__ int first_of(int n, P pred)
{
    const int step = (n + SAE_WAVE - 1) / SAE_WAVE, lane = (int)__lane_id();
    u64 in = __ballot(pred(min((lane + 1) * step, n) - 1));
    if (!in) return n - 1;
    const int from = __builtin_ctzll(in) * step;
    in = __ballot(lane < step && pred(min(from + lane, n - 1)));
    return min(from + __builtin_ctzll(in), n - 1);
}

// Sorts s.list[0 .. n - 1] and fills s.sums with the weights up to each, after `before`.
template <int NW>
__device__ __forceinline__ void sort_and_sum(Shared &s, const Scale &sc, int n, u64 before)
{
    constexpr int THREADS = NW * SAE_WAVE, PER = (LIST + THREADS - 1) / THREADS;
    int size = 2;
    while (size < n) size *= 2;
    for (int i = n + threadIdx.x; i < size; i += THREADS) s.list[i] = ~0ull;
    __syncthreads();
    // a bitonic network, two of its stages at a time
    auto order = [](u64 &a, u64 &b, bool up) {
        const bool swap = (a > b) == up;
        const u64 x = swap ? b : a;
        b = swap ? a : b;
        a = x;
    };
#pragma unroll 1
    for (int k = 2; k <= size; k *= 2) {
        int j = k / 2;
        if (__builtin_ctz(k) & 1) {
            for (int t = threadIdx.x; t < size / 2; t += THREADS) {
                const int i = (t & ~(j - 1)) * 2 + (t & (j - 1));
                u64 a = s.list[i], b = s.list[i + j];
                order(a, b, (i & k) == 0);
                s.list[i] = a;
                s.list[i + j] = b;
            }
            __syncthreads();
            j /= 2;
        }
#pragma unroll 1
        for (; j > 0; j /= 4) {
            const int h = j / 2;
            for (int t = threadIdx.x; t < size / 4; t += THREADS) {
                const int i = (t & ~(h - 1)) * 4 + (t & (h - 1));
                const bool up = (i & k) == 0;
                u64 a = s.list[i], b = s.list[i + h], c = s.list[i + 2 * h], d = s.list[i + 3 * h];
                order(a, c, up);
                order(b, d, up);
                order(a, b, up);
                order(c, d, up);
                s.list[i] = a;
                s.list[i + h] = b;
                s.list[i + 2 * h] = c;
                s.list[i + 3 * h] = d;
            }
            __syncthreads();
        }
    }
    const int per = (n + THREADS - 1) / THREADS, i0 = threadIdx.x * per;
    u64 m[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (i < per && i0 + i < n) sum += sc.weight(logit_of((uint32_t)(s.list[i0 + i] >> 32)));
        m[i] = sum;
    }
    const u64 mb = before + sum_before<NW>(s, 0, sum);
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (i < per && i0 + i < n) s.sums[i0 + i] = mb + m[i];
    __syncthreads();
}

__device__ __forceinline__ u64 uniform64(u64 x) { return (u64)uniform((long long)x); }
__device__ __forceinline__ u64 share(float p, u64 of, bool up)
{
    const double x = (double)p * (double)of;
    return (u64)(up ? __builtin_ceil(x) : __builtin_floor(x));
}
// A token is drawn where the sum passes this.
__device__ __forceinline__ u64 drawn_at(float u, u64 sum) { return u > 0.0f ? min(share(fminf(u, 1.0f), sum, false), sum - 1) : 0; }

// The head of the order that a question asks for: the first `target` tokens where by_count, else the shortest
// whose mass is at least `target`.
struct Head {
    u64 n, mass;
    u64 last;        // weight of its last token
    uint32_t index;  // of its last token (where asked for)
};

template <int DT, int THREADS>
__device__ __forceinline__ Head locate(Shared &s, const Row<DT, THREADS> &row, const Scale &sc, bool by_count, u64 target, bool index)
{
    constexpr int NW = THREADS / SAE_WAVE;
    auto reached = [&](u64 n, u64 mass) { return (by_count ? n : mass) >= target; };
    const int b = first_of(BINS, [&](int i) { return reached(s.bins.count[i], s.bins.mass[i]); });
    u64 n0 = b ? s.bins.count[b - 1] : 0, m0 = b ? s.bins.mass[b - 1] : 0;
    uint32_t left = s.bins.count[b] - (uint32_t)n0;
    if (by_count && b >= LIGHT) return {target, m0, 0, 0};  // (its tokens weigh nothing)
    // tokens of the bin whose keys agree with `key` from bit `shift` on
    const float lo = b >= LIGHT - 1 ? LOWEST : sc.floor_of(b), hi = b < 3 ? __builtin_inff() : sc.floor_of(b - 3);
    uint32_t key = 0;
    int shift = 32;
    auto inside = [&](float l) {
        return l >= lo && l <= hi && l > LOWEST && sc.bin(l) == b && (shift == 32 || key_of(l) >> shift == key >> shift);
    };
    while (left > LIST && shift > 0) {
        const int next = max(shift - 10, 0), mask = (1 << (shift - next)) - 1;
        __syncthreads();
        for (int i = threadIdx.x; i < DIGITS; i += THREADS) {
            s.digits.mass[i] = 0;
            s.digits.count[i] = 0;
        }
        __syncthreads();
        row.each([&](float l, int) {
            if (!inside(l)) return;
            const int d = (int)(key_of(l) >> next) & mask;
            atomicAdd(&s.digits.count[d], 1u);
            atomicAdd(&s.digits.mass[d], sc.weight(l));
        });
        __syncthreads();
        accumulate<NW, DIGITS>(s, s.digits.mass, s.digits.count);
        const int d = first_of(DIGITS, [&](int i) { return reached(n0 + s.digits.count[i], m0 + s.digits.mass[i]); });
        const uint32_t before = d ? s.digits.count[d - 1] : 0;
        left = s.digits.count[d] - before;
        m0 += d ? s.digits.mass[d - 1] : 0;
        n0 += before;
        key |= (uint32_t)d << next;
        shift = next;
    }
    if (left <= LIST) {
        __syncthreads();
        if (threadIdx.x == 0) s.n = 0;
        __syncthreads();
        row.each([&](float l, int i) {
            if (inside(l)) s.list[min(atomicAdd(&s.n, 1u), (uint32_t)LIST - 1)] = (u64)key_of(l) << 32 | (uint32_t)i;
        });
        __syncthreads();
        const int n = uniform((int)s.n);
        sort_and_sum<NW>(s, sc, n, m0);
        const int at = by_count ? min((int)(target - n0), n) - 1 : first_of(n, [&](int i) { return s.sums[i] >= target; });
        const u64 sum = uniform64(s.sums[at]);
        return {n0 + at + 1, sum, sum - (at ? uniform64(s.sums[at - 1]) : m0), (uint32_t)uniform64(s.list[at])};
    }
    // equal logits: their weights are, and they are in order of index
    const u64 w = sc.weight(logit_of(key));
    const u64 r = by_count ? target - n0 : w ? (target - m0 + w - 1) / w : 1;  // how many of them: 1 ..
    Head h = {n0 + r, m0 + r * w, w, 0};
    if (!index) return h;
    uint32_t at = 0, before = 0;
    for (int next = 10; next >= 0; next -= 10) {
        __syncthreads();
        for (int i = threadIdx.x; i < DIGITS; i += THREADS) {
            s.digits.mass[i] = 0;
            s.digits.count[i] = 0;
        }
        __syncthreads();
        row.each([&](float l, int i) {
            if (inside(l) && (next == 10 || (uint32_t)i >> 10 == at >> 10)) atomicAdd(&s.digits.count[i >> next & 1023], 1u);
        });
        __syncthreads();
        accumulate<NW, DIGITS>(s, s.digits.mass, s.digits.count);
        const int d = first_of(DIGITS, [&](int i) { return before + s.digits.count[i] >= r; });
        before += d ? s.digits.count[d - 1] : 0;
        at |= (uint32_t)d << next;
    }
    h.index = at;
    return h;
}

// The answers from the bins that they can lie in; false where those hold too many tokens.
// The questions are asked of the bins first, with bounds in place of the weight that the one before
// leaves: each gives the bins of its answer and bounds for the next one.
template <int DT, int THREADS, typename A>
__device__ __forceinline__ bool answer_in_bins(Shared &s, const Row<DT, THREADS> &row, const Scale &sc, u64 kth, bool whole, float p,
                                               float m, float u, A answer)
{
    constexpr int NW = THREADS / SAE_WAVE;
    auto mass_of = [&](int b) { return b < 0 ? (u64)0 : uniform64(s.bins.mass[b]); };
    auto count_of = [&](int b) { return b < 0 ? 0 : uniform((int)s.bins.count[b]); };
    // the first bin that reached(mass, count) holds for; each lane keeps what is reached every 24 bins
    constexpr int STEP = BINS / SAE_WAVE;
    const int lane = (int)__lane_id();
    const u64 far_mass = s.bins.mass[lane * STEP + STEP - 1];
    const uint32_t far_count = s.bins.count[lane * STEP + STEP - 1];
    auto first_bin = [&](auto reached) __attribute__((always_inline)) {
        u64 in = __ballot(reached(far_mass, far_count));
        if (!in) return BINS - 1;
        const int from = __builtin_ctzll(in) * STEP, i = min(from + lane, BINS - 1);
        in = __ballot(lane < STEP && reached(s.bins.mass[i], s.bins.count[i]));
        return from + (int)__builtin_ctzll(in);
    };
    auto bin_of = [&](u64 mass) { return first_bin([&](u64 x, uint32_t) { return x >= mass; }); };
    int lo[4] = {-2, -2, -2, -2}, hi[4] = {-2, -2, -2, -2};  // of bins; rising and apart in the end
    auto add = [&](int question, int x, int y) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < question; ++i)  // (takes in the ranges that it touches)
            if (lo[i] >= 0 && lo[i] <= y + 1 && x <= hi[i] + 1) {
                x = min(x, lo[i]);
                y = max(y, hi[i]);
                lo[i] = hi[i] = -2;
            }
        lo[question] = x;
        hi[question] = y;
    };
    const u64 all = mass_of(BINS - 1);
    u64 w0 = all, w1 = all;  // bounds of the weight that is left
    int b0 = -1;
    if (!whole) {
        b0 = first_bin([&](u64, uint32_t x) { return x >= kth; });
        w0 = mass_of(b0 - 1);
        w1 = mass_of(b0);
        if (b0 < LIGHT) add(0, b0, b0);
        else w0 = w1;  // (the light bin's tokens weigh nothing)
        w0 = max(w0, (u64)ONE);
    }
    if (p < 1.0f) {
        w0 = max(share(p, w0, true), (u64)ONE);
        const u64 t1 = max(share(p, w1, true), (u64)ONE);
        const int x = bin_of(w0), y = bin_of(t1);
        add(1, x, y);
        w1 = min(w1, mass_of(y));
    }
    int bm = -1;  // bins before bm weigh enough each, bins past bm + 2 do not
    if (m > 0.0f) {
        bm = max((int)fminf(-log2f(fminf(m, 1.0f)) * PER_TWO, (float)LIGHT) - 1, 0);
        add(2, bm, bm + 2);
        w0 = min(w0, max(mass_of(bm - 1), (u64)ONE));
        w1 = min(w1, mass_of(bm + 2));
    }
    {
        const int x = bin_of(drawn_at(u, w0) + 1), y = bin_of(drawn_at(u, w1) + 1);
        add(3, x, y);
    }
    // in order; places in the list, and what lies before them in bins that are not in it
#pragma unroll
    for (int r = 0; r < 3; ++r)
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (lo[i] > lo[i + 1]) {
                const int a = lo[i], b = hi[i];
                lo[i] = lo[i + 1];
                hi[i] = hi[i + 1];
                lo[i + 1] = a;
                hi[i + 1] = b;
            }
    int end = -1;  // lanes 2 i and 2 i + 1: the bins before and at the end of range i
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        end = lane == 2 * i ? lo[i] - 1 : end;
        end = lane == 2 * i + 1 ? hi[i] : end;
    }
    const u64 end_mass = end < 0 ? 0 : s.bins.mass[end];
    const uint32_t end_count = end < 0 ? 0 : s.bins.count[end];
    int at[4], n = 0, behind[4];
    u64 gap[4], held = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // (an empty range: no mass, no tokens)
        at[i] = n;
        behind[i] = (int)of_lane(end_count, 2 * i);
        gap[i] = of_lane(end_mass, 2 * i) - held;
        n += (int)of_lane(end_count, 2 * i + 1) - behind[i];
        held += of_lane(end_mass, 2 * i + 1) - of_lane(end_mass, 2 * i);
    }
    if (n > LIST) return false;
    __syncthreads();
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    // the ranges' logits: from the lowest of its bins to below the lowest of the bins before
    for (int t = threadIdx.x / SAE_WAVE; t < 8; t += NW) {
        const int b = t & 1 ? lo[t / 2] - 1 : hi[t / 2];
        const float x = lo[t / 2] < 0 ? __builtin_inff() : b < 0 ? __builtin_inff() : b >= LIGHT ? -0x1.fffffep127f : lowest_of(sc, b);
        if (__lane_id() == 0) s.edges[t] = x;
    }
    __syncthreads();
    float least[4], past[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        least[j] = s.edges[2 * j];
        past[j] = s.edges[2 * j + 1];
    }
    // (what lies between several ranges collected too and sifted in LDS, where it is little: no faster)
    uint32_t *indexes = reinterpret_cast<uint32_t *>(s.sums);
    if (lo[2] < 0)  // uniform: one range
        row.collect(indexes, &s.n, LIST, [&](float l) { return (l >= least[3]) & (l < past[3]); });
    else if (lo[1] < 0)  // two
        row.collect(indexes, &s.n, LIST, [&](float l) { return ((l >= least[2]) & (l < past[2])) | ((l >= least[3]) & (l < past[3])); });
    else
        row.collect(indexes, &s.n, LIST, [&](float l) {
            return ((l >= least[0]) & (l < past[0])) | ((l >= least[1]) & (l < past[1])) | ((l >= least[2]) & (l < past[2])) |
                   ((l >= least[3]) & (l < past[3]));
        });
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS) s.list[i] = (u64)key_of(row.logit((int)indexes[i])) << 32 | indexes[i];
    __syncthreads();
    sort_and_sum<NW>(s, sc, n, 0);
    for (int i = threadIdx.x; i < n; i += THREADS) {
        u64 g = gap[0];
#pragma unroll
        for (int j = 1; j < 4; ++j) g = lo[j] >= 0 && i >= at[j] ? gap[j] : g;
        s.sums[i] += g;
    }
    __syncthreads();
    auto weight_at = [&](int i) { return sc.weight(logit_of((uint32_t)(s.list[i] >> 32))); };
    // tokens of the order before the list's token i
    auto before = [&](int i) {
        int b = 0, first = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (lo[j] >= 0 && i >= at[j]) {
                b = behind[j];
                first = at[j];
            }
        return b + i - first;
    };
    u64 kept = kth, w = all;
    if (!whole) {
        if (b0 >= LIGHT) w = all;
        else {
            int i = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (lo[j] >= 0 && lo[j] <= b0) i = at[j] + (int)kth - 1 - behind[j];
            w = uniform64(s.sums[i]);
        }
    }
    if (p < 1.0f) {
        const u64 target = max(share(p, w, true), 1ull);
        const int i = first_of(n, [&](int i) { return s.sums[i] >= target; });
        w = uniform64(s.sums[i]);
        kept = before(i) + 1;
    }
    if (m > 0.0f) {
        const double least = (double)m * ONE;
        int from = 0, to = 0;  // the list's tokens of bins bm .. bm + 2
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (lo[j] >= 0 && lo[j] <= bm && hi[j] >= bm + 2) {
                from = at[j] + count_of(bm - 1) - behind[j];
                to = at[j] + count_of(bm + 2) - behind[j];
            }
        __syncthreads();
        if (threadIdx.x == 0) s.found = to;
        __syncthreads();
        for (int i = from + threadIdx.x; i < to; i += THREADS)
            if ((double)weight_at(i) < least) atomicMin(&s.found, (uint32_t)i);
        __syncthreads();
        const int i = uniform((int)s.found);  // the first that weighs too little
        u64 c = count_of(bm - 1) + i - from, mass = i > from ? uniform64(s.sums[i - 1]) : mass_of(bm - 1);
        if (c == 0) {
            c = 1;
            mass = (u64)ONE;
        }
        if (c < kept) {
            kept = c;
            w = mass;
        }
    }
    const u64 target = drawn_at(u, w);
    const int i = first_of(n, [&](int i) { return s.sums[i] > target; });
    if (threadIdx.x == 0) answer((uint32_t)s.list[i], (float)((double)weight_at(i) / (double)w), (uint32_t)kept);
    return true;
}

struct Settings {
    float T, p, m, u;
    int k;
    __device__ __forceinline__ Settings(const Args &a, int r)
        : T(a.temperature ? a.temperature[r] : 1.0f), p(a.top_p ? a.top_p[r] : 1.0f), m(a.min_p ? a.min_p[r] : 0.0f), u(a.u[r]),
          k(a.top_k ? a.top_k[r] : 0)
    {
    }
    __device__ __forceinline__ bool greedy() const { return !(T > 0.0f) || k == 1 || p <= 0.0f; }
    // Of mapped() logits: at T = 1 the ones below the largest weigh nothing (a T past 5e36 would leave them something).
    __device__ __forceinline__ void set_infinite() { T = T > 0.0f ? 1.0f : T; }
};
template <int THREADS>
constexpr int SMALL_K = THREADS / 2;  // a k that the threads' maxima bound (256 rows of 131,072, k 300: 25.9 us, by the histogram 76.4)

__device__ __forceinline__ Scale scale_of_row(float top, float T, const double *power)
{
    return {(double)top, PER_TWO * 1.44269504088896340736 / (double)T, power};
}
__device__ __forceinline__ void fill_powers(Shared &s)
{
    if (threadIdx.x < PER_TWO) s.power[threadIdx.x] = __builtin_ldexp(exp2(threadIdx.x * (-1.0 / PER_TWO)), 43);
}

// The first launch of few rows: maxima of the row's groups, 256 a workgroup, and an empty histogram.
template <int DT>
__global__ void __launch_bounds__(256) k_draw_max(Args a)
{
    __shared__ float part[4];
    const int r = blockIdx.y;
    const Row<DT, 256> row(static_cast<const char *>(a.logits) + (int64_t)r * a.stride * Row<DT, 256>::SIZE, a.vocab);
    Shelf &shelf = reinterpret_cast<Shelf *>(a.work)[r];
    const int g = blockIdx.x * 256 + threadIdx.x;
    for (int i = g; i < BINS; i += gridDim.x * 256) {
        shelf.mass[i] = 0;
        shelf.count[i] = 0;
    }
    float m = LOWEST;
    for (int v = g; v < row.vectors; v += SPLIT_GROUPS) {
        const u32x4 x = row.vector(v);
#pragma unroll
        for (int i = 0; i < Row<DT, 256>::E; ++i) m = fmaxf(m, row.wide(x, i));
    }
    if (g < SPLIT_GROUPS) shelf.most[g] = m;
    m = upto(m, LOWEST, [](float x, float y) { return fmaxf(x, y); });
    if (__lane_id() == SAE_WAVE - 1) part[threadIdx.x / SAE_WAVE] = m;
    __syncthreads();
    if (threadIdx.x == 0) shelf.maxes[blockIdx.x] = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
}

// The second: a part of the row's vectors into the histogram.
template <int DT>
__global__ void __launch_bounds__(512) k_draw_hist(Args a, int maxes)
{
    __shared__ Shared s;
    const int r = blockIdx.y;
    Settings set(a, r);
    if (set.greedy()) return;  // uniform: not asked for
    Row<DT, 512> row(static_cast<const char *>(a.logits) + (int64_t)r * a.stride * Row<DT, 512>::SIZE, a.vocab);
    Shelf &shelf = reinterpret_cast<Shelf *>(a.work)[r];
    fill_powers(s);
    for (int i = threadIdx.x; i < BINS; i += 512) {
        s.bins.mass[i] = 0;
        s.bins.count[i] = 0;
    }
    row.load_edge();
    const float mine = (int)threadIdx.x < maxes ? fmaxf(shelf.maxes[threadIdx.x], row.edge) : row.edge;
    const float top = over_all<8>(s, 0, mine, LOWEST, [](float x, float y) { return fmaxf(x, y); });
    if (!(top > LOWEST)) return;
    if (top == __builtin_inff()) {
        row.infinite = true;
        row.edge = row.mapped(row.edge);
        set.set_infinite();
    }
    const Scale sc = scale_of_row(row.infinite ? 0.0f : top, set.T, s.power);
    uint32_t light = 0;
    auto put = [&](float l, int) {
        double rest;
        const int b = sc.split(l, rest);
        if (b < LIGHT) {
            atomicAdd(&s.bins.count[b], 1u);
            atomicAdd(&s.bins.mass[b], sc.weight(b, rest));
        } else {
            light += l > LOWEST;
        }
    };
    const int per = (row.vectors + (int)gridDim.x - 1) / (int)gridDim.x, first = min((int)blockIdx.x * per, row.vectors);
    row.each_of(first, min(first + per, row.vectors), sc.floor_of(LIGHT), put, [&](float l) { light += l > LOWEST; });
    if (blockIdx.x == 0 && row.edge_at >= 0) put(row.edge, row.edge_at);
    light = sum_upto(light);
    if (__lane_id() == SAE_WAVE - 1 && light) atomicAdd(&s.bins.count[LIGHT], light);
    __syncthreads();
    for (int i = threadIdx.x; i < BINS; i += 512)
        if (s.bins.count[i]) {
            atomicAdd(&shelf.count[i], s.bins.count[i]);
            if (s.bins.mass[i]) atomicAdd(&shelf.mass[i], s.bins.mass[i]);
        }
}

// (Four waves a SIMD, two workgroups of 512 a compute unit: 700 rows of 50,001 at 130 registers 90 us, at 120 72.5.)
template <int DT, int THREADS, bool SPLIT>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 3 : 4) k_draw(Args a)
{
    constexpr int NW = THREADS / SAE_WAVE;
    __shared__ Shared s;
    const int r = blockIdx.x, lane = (int)__lane_id(), wave = threadIdx.x / SAE_WAVE;
    Row<DT, THREADS> row(static_cast<const char *>(a.logits) + (int64_t)r * a.stride * Row<DT, THREADS>::SIZE, a.vocab);
    Settings set(a, r);
    const float p = set.p, m = set.m, u = set.u;
    const int k = SPLIT ? 0 : set.k;  // (rows with a top_k are not split)
    auto answer = [&](uint32_t token, float prob, uint32_t kept) {
        a.token[r] = (int32_t)token;
        if (a.prob) a.prob[r] = prob;
        if (a.kept) a.kept[r] = (int32_t)kept;
    };
    const Shelf *const shelf = SPLIT ? reinterpret_cast<const Shelf *>(a.work) + r : nullptr;
    fill_powers(s);
    float mine;
    if constexpr (SPLIT) mine = row.maxima_of(*shelf);
    else mine = row.maxima();
    float top = over_all<NW>(s, 0, mine, LOWEST, [](float x, float y) { return fmaxf(x, y); });
    if (!(top > LOWEST)) {
        if (threadIdx.x == 0) answer(~0u, 0.0f, 0);
        return;
    }
    if (top == __builtin_inff()) {  // uniform
        row.set_infinite();
        mine = row.mapped(mine);
        top = 0.0f;
        set.set_infinite();
    }
    if (set.greedy()) {  // the first of the largest
        uint32_t first = ~0u;
        row.some(top, [&](float l, int i) {
            if (l == top) first = min(first, (uint32_t)i);
        });
        first = over_all<NW>(s, 1, first, ~0u, [](uint32_t x, uint32_t y) { return min(x, y); });
        if (threadIdx.x == 0) answer(first, 1.0f, 1);
        return;
    }
    const Scale sc = scale_of_row(top, set.T, s.power);

    // the list: the first tokens of the order, enough of them for every question
    int n = LIST + 1;    // in the list; more than LIST: not collected
    bool whole = false;  // `total` is the weight of all tokens, and top-k leaves them all
    u64 total = 0;
    if (!SPLIT && k > 0 && k <= SMALL_K<THREADS>) {
        // the k-th largest of the threads' maxima, to 16 bits of its key; every wave finds it by itself
        uint32_t bound = 0, want = (uint32_t)k;
        const uint32_t key = key_of(mine);
        for (int i = threadIdx.x; i < 512; i += THREADS) s.digits.count[i] = 0;
        if (threadIdx.x == 0) s.n = 0;
        __syncthreads();
#pragma unroll 1
        for (int shift = 24; shift >= 16; shift -= 8) {
            uint32_t *const count = s.digits.count + (shift == 16 ? 256 : 0);
            if (shift == 24 || key >> 24 == bound >> 24) atomicAdd(&count[key >> shift & 255], 1u);
            __syncthreads();
            uint32_t c[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                c[i] = count[lane * 4 + i];
                sum += c[i];
            }
            uint32_t before = sum_upto(sum) - sum;
            const int at = __builtin_ctzll(__ballot(before < want && before + sum >= want));
            uint32_t digit = lane * 4;
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                const bool past = digit == (uint32_t)(lane * 4 + i) && before + c[i] < want;
                before += past ? c[i] : 0;
                digit += past;
            }
            bound |= of_lane(digit, at) << shift;
            want -= of_lane(before, at);
        }
        const float least = fmaxf(logit_of(bound | 0xFFFFu), -0x1.fffffep127f);  // (-inf is not taken)
        row.some(least, [&](float l, int i) {
            if (l >= least) {
                const uint32_t at = atomicAdd(&s.n, 1u);
                if (at < LIST) s.list[at] = (u64)key_of(l) << 32 | (uint32_t)i;
            }
        });
        __syncthreads();
        n = uniform((int)s.n);
    }
    u64 kth = 0;  // tokens that top-k leaves
    if (n > LIST) {
        __syncthreads();
        for (int i = threadIdx.x; i < BINS; i += THREADS) {
            s.bins.mass[i] = SPLIT ? shelf->mass[i] : 0;
            s.bins.count[i] = SPLIT ? shelf->count[i] : 0;
        }
        if (threadIdx.x == 0) s.n = 0;
        __syncthreads();
        uint32_t light = 0;
        if constexpr (!SPLIT)
            row.each(row.any_below(sc.floor_of(LIGHT)),
                     [&](float l, int) {
                         double rest;
                         const int b = sc.split(l, rest);
                         if (b < LIGHT) {
                             atomicAdd(&s.bins.count[b], 1u);
                             atomicAdd(&s.bins.mass[b], sc.weight(b, rest));
                         } else {
                             light += l > LOWEST;
                         }
                     },
                     [&](float l) { light += l > LOWEST; });
        light = sum_upto(light);
        if (lane == SAE_WAVE - 1 && light) atomicAdd(&s.bins.count[LIGHT], light);
        __syncthreads();
        accumulate<NW, BINS>(s, s.bins.mass, s.bins.count);
        const uint32_t all = s.bins.count[BINS - 1];
        total = s.bins.mass[BINS - 1];
        kth = k > 0 && (uint32_t)k < all ? (uint32_t)k : all;
        whole = kth == all;
        int last = whole ? LIGHT : first_of(BINS, [&](int i) { return s.bins.count[i] >= kth; });
        // (top-p of what top-k leaves: its weight has to be known first)
        if (whole && p < 1.0f) {
            const u64 most = share(p, total, true);
            last = first_of(BINS, [&](int i) { return s.bins.mass[i] >= most; });
        }
        if (m > 0.0f && (whole || !(p < 1.0f))) {
            const float x = -log2f(fminf(m, 1.0f)) * PER_TWO + 2.0f;
            if (x < (float)last) last = (int)x;
        }
        n = (int)s.bins.count[last];
        if (n <= SAE_WAVE) {
            const float least = last >= LIGHT - 1 ? -0x1.fffffep127f : sc.floor_of(last);
            row.some(least, [&](float l, int i) {
                if (l >= least && sc.bin(l) <= last) s.list[min(atomicAdd(&s.n, 1u), (uint32_t)LIST - 1)] = (u64)key_of(l) << 32 | (uint32_t)i;
            });
            __syncthreads();
        } else if (answer_in_bins(s, row, sc, kth, whole, p, m, u, answer)) {
            return;
        } else {
            n = LIST + 1;
        }
    }
    if (n <= SAE_WAVE) {  // one wave, a token a lane
        // ranks: each wave counts what of its part of the list comes before a token
        u64 item = lane < n ? s.list[lane] : ~0ull;
        u32x4 *const counts = reinterpret_cast<u32x4 *>(s.sums);  // a byte a wave for each token
        uint32_t rank = 0;
#pragma unroll
        for (int i = 0; i < SAE_WAVE / NW; ++i) {
            const int j = wave * (SAE_WAVE / NW) + i;
            rank += j < n && s.list[j] < item;
        }
        reinterpret_cast<uint8_t *>(counts + lane)[wave] = (uint8_t)rank;
        __syncthreads();
        if (wave != 0) return;
        const u32x4 c = counts[lane];
        rank = 0;
#pragma unroll
        for (int i = 0; i < NW / 4; ++i) rank = __builtin_amdgcn_sad_u8(c[i], 0, rank);
        if (lane < n) s.list[rank] = item;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        item = s.list[lane];
        const u64 w = lane < n ? sc.weight(logit_of((uint32_t)(item >> 32))) : 0, sum = sum_upto(w);
        int keep = k > 0 ? min(k, n) : n;
        auto first = [&](bool x) { return __builtin_ctzll(__ballot(x) | 1ull << (keep - 1)); };
        if (p < 1.0f) {
            const u64 target = share(p, whole ? total : of_lane(sum, keep - 1), true);
            keep = first(sum >= target) + 1;
        }
        if (m > 0.0f) {
            const double least = (double)m * ONE;
            const u64 light = __ballot(lane < n && (double)w < least);
            if (light) keep = max(min(keep, __builtin_ctzll(light)), 1);
        }
        const u64 of = of_lane(sum, keep - 1), target = drawn_at(u, of);
        const int at = first(sum > target);
        if (lane == at) answer((uint32_t)item, (float)((double)w / (double)of), keep);
        return;
    }
    if (n <= LIST) {
        sort_and_sum<NW>(s, sc, n, 0);
        int keep = k > 0 ? min(k, n) : n;
        if (p < 1.0f) {
            const u64 target = share(p, whole ? total : uniform64(s.sums[keep - 1]), true);
            keep = first_of(keep, [&](int i) { return s.sums[i] >= target; }) + 1;
        }
        if (m > 0.0f) {
            const double least = (double)m * ONE;
            auto light = [&](int i) { return (double)(s.sums[i] - (i ? s.sums[i - 1] : 0)) < least; };
            const int at = first_of(keep, light);
            if (light(at)) keep = max(at, 1);
        }
        const u64 of = uniform64(s.sums[keep - 1]), target = drawn_at(u, of);
        const int at = first_of(keep, [&](int i) { return s.sums[i] > target; });
        if (threadIdx.x == 0) answer((uint32_t)s.list[at], (float)((double)(s.sums[at] - (at ? s.sums[at - 1] : 0)) / (double)of), keep);
        return;
    }
    // too many for the list: each question by itself
    Head h = {kth, total, 0, 0};
#pragma unroll 1
    for (int question = 0;; ++question) {  // top-k, top-p, min-p, the token
        if ((question == 0 && whole) || (question == 1 && !(p < 1.0f)) || (question == 2 && !(m > 0.0f))) continue;
        if (question != 2) {
            const u64 target = question == 0 ? kth : question == 1 ? max(share(p, h.mass, true), 1ull) : drawn_at(u, h.mass) + 1;
            const Head found = locate(s, row, sc, question == 0, target, question == 3);
            if (question == 3) {
                if (threadIdx.x == 0) answer(found.index, (float)((double)found.last / (double)h.mass), (uint32_t)h.n);
                return;
            }
            h = found;
            continue;
        }
        const double least = (double)m * ONE;
        uint32_t c = 0;
        u64 mass = 0;
        row.each([&](float l, int) {
            const u64 w = sc.weight(l);
            const bool in = (double)w >= least && l > LOWEST;
            c += in;
            mass += in ? w : 0;
        });
        __syncthreads();
        const uint32_t c_all = over_all<NW>(s, 0, c, 0u, [](uint32_t x, uint32_t y) { return x + y; });
        const u64 m_all = over_all<NW>(s, 1, mass, (u64)0, [](u64 x, u64 y) { return x + y; });
        if (c_all == 0) h = {1, (u64)ONE, 0, 0};  // (min-p above 1)
        else if (c_all < h.n) h = {c_all, m_all, 0, 0};
    }
}

// Rows whose passes are launches of their own: from 65,536 tokens and to 64 rows (one row of 131,072 bf16 logits
// with top-p: 47.0 us as one launch, 26.4 as three; 64 rows 70.9 and 58.1; 64 rows of 64,000 43.7 and 43.4, 200
// rows of 131,072 81.5 and 94.1), but not with a top_k: rows with a small k read theirs once (14.6 us instead of 10.3).
constexpr int SPLIT_VOCAB = 65536, SPLIT_ROWS = 64;
bool is_split(int rows, int vocab) { return vocab >= SPLIT_VOCAB && rows <= SPLIT_ROWS; }

template <int DT>
void launch(const Args &a, int rows, hipStream_t s)
{
    if (is_split(rows, a.vocab) && !a.top_k) {
        const int vectors = a.vocab / Row<DT, 256>::E, maxes = std::min((vectors + 255) / 256, SPLIT_MAXES);
        hipLaunchKernelGGL((k_draw_max<DT>), dim3(maxes, rows), dim3(256), 0, s, a);
        // about two workgroups per compute unit, of at least 4 vectors a thread
        const int parts = std::max(std::min(512 / rows, vectors / 2048), 1);
        hipLaunchKernelGGL((k_draw_hist<DT>), dim3(parts, rows), dim3(512), 0, s, a, maxes);
        hipLaunchKernelGGL((k_draw<DT, 1024, true>), dim3(rows), dim3(1024), 0, s, a);
        return;
    }
    // Threads of a row (bf16 logits, top-p, us with 256 / 512 / 1,024: 600 rows of 4,000 17.3 / 22.7 / 37.4, of 8,192 21.5 /
    // 26.2 / 44.9; 64 rows of 4,000 13.6 / 13.8 / 17.9; 300 rows of 16,000 26.1 / 24.5 / 34.7, of 50,000 57.9 / 52.3 /
    // 59.5; 64 rows of 16,000 22.9 / 18.8 / 23.3, of 32,000 34.2 / 26.0 / 28.1; one row of 16,000 16.4 / 13.3 / 14.7, of
    // 50,000 35.7 / 25.7 / 24.5; with 512 / 1,024: 256 rows of 131,072 82.7 / 76.4, 400 rows 115.9 / 130.9, with settings by
    // row 159 / 135).
    const bool half = rows >= 512 || a.vocab <= 16384 || (rows > 16 && a.vocab < 65536);
    if (a.vocab <= 8192) hipLaunchKernelGGL((k_draw<DT, 256, false>), dim3(rows), dim3(256), 0, s, a);
    else if (half) hipLaunchKernelGGL((k_draw<DT, 512, false>), dim3(rows), dim3(512), 0, s, a);
    else hipLaunchKernelGGL((k_draw<DT, 1024, false>), dim3(rows), dim3(1024), 0, s, a);
}

}  // namespace

// (More rows are not split, but a workspace that was made for them serves fewer ones, which are.)
size_t sample_work_bytes(int rows, int vocab)
{
    return rows > 0 && vocab >= SPLIT_VOCAB ? std::min(rows, SPLIT_ROWS) * sizeof(Shelf) : 16;
}

hipError_t launch_sample(int rows, int vocab, int dtype, const SampleArgs &x, hipStream_t s)
{
    const Args a = {x.logits, x.stride, x.settings.temperature, x.settings.top_p, x.settings.min_p, x.u, x.settings.top_k,
                    x.token, x.kept, x.prob, vocab, static_cast<char *>(x.work)};
    if (dtype == SAE_KV_BF16) launch<SAE_KV_BF16>(a, rows, s);
    else if (dtype == SAE_KV_F16) launch<SAE_KV_F16>(a, rows, s);
    else launch<SAE_ROWS_F32>(a, rows, s);
    return hipGetLastError();
}
