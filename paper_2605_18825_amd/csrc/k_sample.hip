// Sampling a token per row of logits by temperature, top-k, top-p and min-p.
//
// Every part of the definition is a question to one order, by falling logit and rising index: the
// weight of its first k tokens, the shortest head that holds p of it, the token where u of it is
// passed.  So nothing is sorted but the few tokens that the answers lie among.  Weights
// exp((l - l_0) / T) are computed in 64 bits and held as whole multiples of 2^-43 (the sum of 2^20
// fits 64 bits): sums are exact, whatever their order, and LDS atomics can take them.
//
// A workgroup takes a row.
//   small k     the k-th largest of the threads' maxima bounds the k-th largest logit from below:
//               one more pass collects what is not below it, a few more than k tokens.
//   otherwise   a histogram over (l_0 - l) / T, 64 bins per unit, holds each bin's tokens and
//               weight; the answers' bin follows from it, and one more pass collects the tokens up
//               to that bin.
//   where these are more than LDS holds, each question is answered by itself: its bin, then
//   (a bin of many equal or near logits) 11 bits of the logit at a time, then the index.
#include "attn_tile.h"

namespace {

using attn::scan;
using attn::uniform;

constexpr int NW = 16, THREADS = NW * SAE_WAVE;
constexpr int LIST = 2048;           // tokens that are sorted in LDS
constexpr int BINS = 2048;           // of a histogram; the last one's tokens weigh nothing
constexpr float PER_UNIT = 64.0f;    // bins of a unit of (l_0 - l) / T: 2047 / 64 = 32 units, e^-32 = 2^-46
constexpr int SMALL_K = 256;         // threads' maxima bound the k-th logit
constexpr double ONE = 8796093022208.0;  // 2^43
typedef unsigned long long u64;

struct Args {
    const void *logits;
    int64_t stride;
    const float *temperature, *top_p, *min_p, *u;
    const int32_t *top_k;
    int32_t *token, *kept;
    float *prob;
    int32_t vocab;
};

// Ascending whole numbers for falling logits.
__device__ __forceinline__ uint32_t key_of(float l)
{
    const uint32_t b = __float_as_uint(l + 0.0f);  // (-0 and 0 are equal)
    return b >> 31 ? b : ~b & 0x7FFFFFFFu;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key >> 31 ? key : ~key & 0x7FFFFFFFu); }

template <int DT>
struct Row {
    static constexpr int E = DT == SAE_ROWS_F32 ? 4 : 8;  // logits of 16 bytes
    static constexpr int SIZE = 16 / E;
    const char *at;
    int n, head, vectors;  // logits before the first 16-byte boundary, whole vectors behind them

    __device__ __forceinline__ Row(const void *p, int vocab) : at(static_cast<const char *>(p)), n(vocab)
    {
        head = min((int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / SIZE, n);
        vectors = (n - head) / E;
    }
    static __device__ __forceinline__ float wide(u32x4 x, int i)
    {
        if constexpr (DT == SAE_ROWS_F32) return __uint_as_float(x[i]);
        else return i & 1 ? attn::high<DT == SAE_KV_F16>(x[i / 2]) : attn::low<DT == SAE_KV_F16>(x[i / 2]);
    }
    __device__ __forceinline__ float one(int i) const
    {
        if constexpr (DT == SAE_ROWS_F32) return reinterpret_cast<const float *>(at)[i];
        else return attn::low<DT == SAE_KV_F16>((uint32_t)reinterpret_cast<const uint16_t *>(at)[i]);
    }
    // f(logit, index) for every logit, by the whole workgroup.
    template <typename F>
    __device__ __forceinline__ void each(F f) const
    {
        constexpr int UN = 4;
        const char *body = at + (int64_t)head * SIZE;
        const int t = threadIdx.x;
#pragma unroll 1
        for (int v = t; v < vectors; v += THREADS * UN) {
            u32x4 x[UN];
#pragma unroll
            for (int k = 0; k < UN; ++k) {
                const int w = min(v + k * THREADS, vectors - 1);
                x[k] = *reinterpret_cast<const u32x4 *>(body + (int64_t)w * 16);
            }
#pragma unroll
            for (int k = 0; k < UN; ++k)
                if (v + k * THREADS < vectors) {
#pragma unroll
                    for (int i = 0; i < E; ++i) f(wide(x[k], i), head + (v + k * THREADS) * E + i);
                }
        }
        const int tail = n - head - vectors * E;  // fewer than E, as the head's
        if (t < head) f(one(t), t);
        else if (t >= SAE_WAVE && t < SAE_WAVE + tail) f(one(n - tail + t - SAE_WAVE), n - tail + t - SAE_WAVE);
    }
};

template <typename T, typename F>
__device__ __forceinline__ T over_wave(T x, F f)
{
#pragma unroll
    for (int o = 1; o < SAE_WAVE; o <<= 1) x = f(x, __shfl_xor(x, o));
    return x;
}

struct Hist {
    u64 mass[BINS];
    uint32_t count[BINS];
};

struct Shared {
    Hist bins;
    union {           // (digits are done with when a list is summed)
        Hist digits;
        u64 sums[LIST];  // weights up to each token of the list, itself included
    };
    u64 list[LIST];   // key << 32 | index
    u64 tmp[NW];
    uint32_t tmp32[NW];
    uint32_t n, found;
};

// A row's weights and bins.
struct Scale {
    float top, bins_per;  // l_0; bins of a unit of l_0 - l
    double c;             // log2 e / T

    // 2^((l - l_0) c) in units of 2^-43, by the Taylor series of its fractional part (next term 6e-15).
    __device__ __forceinline__ u64 weight(float l) const
    {
        if (l == top) return (u64)ONE;
        if (top == __builtin_inff()) return 0;
        const double z = ((double)l - (double)top) * c;
        if (!(z > -46.0)) return 0;
        const double n = __builtin_rint(z), f = (z - n) * 0.693147180559945309417;
        double y = 1.0 / 39916800;
        y = __builtin_fma(y, f, 1.0 / 3628800);
        y = __builtin_fma(y, f, 1.0 / 362880);
        y = __builtin_fma(y, f, 1.0 / 40320);
        y = __builtin_fma(y, f, 1.0 / 5040);
        y = __builtin_fma(y, f, 1.0 / 720);
        y = __builtin_fma(y, f, 1.0 / 120);
        y = __builtin_fma(y, f, 1.0 / 24);
        y = __builtin_fma(y, f, 1.0 / 6);
        y = __builtin_fma(y, f, 0.5);
        y = __builtin_fma(y, f, 1.0);
        y = __builtin_fma(y, f, 1.0);
        // rounded to a whole number by 2^52, whose last bit is 1
        const double w = __builtin_ldexp(y, (int)n + 43) + 4503599627370496.0;
        return (u64)__double_as_longlong(w) & 0xFFFFFFFFFFFFFull;
    }
    // Rises as l falls; the last one for tokens that weigh nothing (and others as light).
    __device__ __forceinline__ int bin(float l) const
    {
        if (l == top) return 0;
        if (top == __builtin_inff()) return BINS - 1;
        const float x = fminf(top - l, 3.4028235e38f) * bins_per;
        return x < (float)(BINS - 1) ? (int)x : BINS - 1;
    }
};

__device__ __forceinline__ void clear(Hist &h)
{
    for (int i = threadIdx.x; i < BINS; i += THREADS) {
        h.mass[i] = 0;
        h.count[i] = 0;
    }
}

// Counts and masses up to each bin, itself included.
__device__ __forceinline__ void accumulate(Shared &s, Hist &h)
{
    static_assert(BINS == 2 * THREADS, "two bins a thread");
    const int i = threadIdx.x * 2;
    const uint32_t c0 = h.count[i], c1 = h.count[i + 1];
    const u64 m0 = h.mass[i], m1 = h.mass[i + 1];
    uint32_t ct;
    u64 mt;
    const uint32_t c = scan<NW>(c0 + c1, ct, s.tmp32);
    const u64 m = scan<NW>(m0 + m1, mt, s.tmp);
    h.count[i] = c + c0;
    h.count[i + 1] = c + c0 + c1;
    h.mass[i] = m + m0;
    h.mass[i + 1] = m + m0 + m1;
    __syncthreads();
}

// The first bin up to which `pred(count, mass)` holds (it stays true from there on); BINS - 1 where none is.
template <typename P>
__device__ __forceinline__ int first_bin(Shared &s, const Hist &h, P pred)
{
    __syncthreads();
    if (threadIdx.x == 0) s.found = BINS - 1;
    __syncthreads();
    for (int i = threadIdx.x; i < BINS; i += THREADS)
        if (pred(h.count[i], h.mass[i]) && (i == 0 || !pred(h.count[i - 1], h.mass[i - 1]))) s.found = i;
    __syncthreads();
    return uniform((int)s.found);
}

// Sorts s.list[0 .. n - 1] and fills s.sums with the weights up to each, after `before`.
__device__ __forceinline__ void sort_and_sum(Shared &s, const Scale &sc, int n, u64 before)
{
    int size = 2;
    while (size < n) size *= 2;
    for (int i = n + threadIdx.x; i < size; i += THREADS) s.list[i] = ~0ull;
    __syncthreads();
#pragma unroll 1
    for (int k = 2; k <= size; k *= 2)
#pragma unroll 1
        for (int j = k / 2; j > 0; j /= 2) {
            const int i = threadIdx.x / j * 2 * j + threadIdx.x % j;
            if (i < size) {
                const u64 a = s.list[i], b = s.list[i + j];
                if ((a > b) == ((i & k) == 0)) {
                    s.list[i] = b;
                    s.list[i + j] = a;
                }
            }
            __syncthreads();
        }
    const int i = threadIdx.x * 2;
    const u64 a = i < n ? sc.weight(logit_of((uint32_t)(s.list[i] >> 32))) : 0;
    const u64 b = i + 1 < n ? sc.weight(logit_of((uint32_t)(s.list[i + 1] >> 32))) : 0;
    u64 total;
    const u64 m = before + scan<NW>(a + b, total, s.tmp);
    if (i < n) s.sums[i] = m + a;
    if (i + 1 < n) s.sums[i + 1] = m + a + b;
    __syncthreads();
}

// The number of the list's tokens before the first one for which pred(sum up to it) holds.
template <typename P>
__device__ __forceinline__ int first_sum(Shared &s, int n, P pred)
{
    __syncthreads();
    if (threadIdx.x == 0) s.found = n;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS)
        if (pred(s.sums[i]) && (i == 0 || !pred(s.sums[i - 1]))) s.found = i;
    __syncthreads();
    return uniform((int)s.found);
}

__device__ __forceinline__ u64 uniform64(u64 x) { return (u64)uniform((long long)x); }

// The head of the order that a question asks for, when its tokens are not in the list: the first
// n tokens where BY_COUNT (target = n), else the shortest whose mass is at least target.
struct Head {
    u64 n, mass;
    u64 last;         // weight of its last token
    uint32_t index;   // of its last token (where asked for)
};

template <int DT>
__device__ __forceinline__ Head locate(Shared &s, const Row<DT> &row, const Scale &sc, bool by_count, u64 target, bool index)
{
    auto reached = [&](u64 n, u64 mass) { return (by_count ? n : mass) >= target; };
    const int b = first_bin(s, s.bins, [&](uint32_t n, u64 mass) { return reached(n, mass); });
    u64 n0 = b ? s.bins.count[b - 1] : 0, m0 = b ? s.bins.mass[b - 1] : 0;
    uint32_t left = s.bins.count[b] - (uint32_t)n0;
    // tokens of the bin whose keys agree with `key` above bit `shift`
    uint32_t key = 0;
    int shift = 32;
    auto inside = [&](float l) {
        return l > attn::NEG_INF && sc.bin(l) == b && (shift == 32 || key_of(l) >> shift == key >> shift);
    };
    while (left > LIST && shift > 0) {
        const int bits = shift == 32 ? 11 : min(shift, 11), next = shift - bits;
        __syncthreads();
        clear(s.digits);
        __syncthreads();
        row.each([&](float l, int) {
            if (!inside(l)) return;
            const int d = (int)(key_of(l) >> next) & ((1 << bits) - 1);
            atomicAdd(&s.digits.count[d], 1u);
            atomicAdd(&s.digits.mass[d], sc.weight(l));
        });
        __syncthreads();
        accumulate(s, s.digits);
        const int d = first_bin(s, s.digits, [&](uint32_t n, u64 mass) { return reached(n0 + n, m0 + mass); });
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
        sort_and_sum(s, sc, n, m0);
        const int at = by_count ? min((int)(target - n0), n) - 1 : min(first_sum(s, n, [&](u64 sum) { return sum >= target; }), n - 1);
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
        clear(s.digits);
        __syncthreads();
        row.each([&](float l, int i) {
            if (inside(l) && (next == 10 || (uint32_t)i >> 10 == at >> 10)) atomicAdd(&s.digits.count[i >> next & 1023], 1u);
        });
        __syncthreads();
        accumulate(s, s.digits);
        const int d = first_bin(s, s.digits, [&](uint32_t n, u64) { return before + n >= r; });
        before += d ? s.digits.count[d - 1] : 0;
        at |= (uint32_t)d << next;
    }
    h.index = at;
    return h;
}

__device__ __forceinline__ u64 share(float p, u64 of, bool up)
{
    const double x = (double)p * (double)of;
    return (u64)(up ? __builtin_ceil(x) : __builtin_floor(x));
}

template <int DT>
__global__ void __launch_bounds__(THREADS) k_sample(Args a)
{
    __shared__ Shared s;
    const int r = blockIdx.x, lane = (int)__lane_id(), wave = threadIdx.x / SAE_WAVE;
    const Row<DT> row(static_cast<const char *>(a.logits) + (int64_t)r * a.stride * Row<DT>::SIZE, a.vocab);
    const float T = a.temperature ? a.temperature[r] : 1.0f, p = a.top_p ? a.top_p[r] : 1.0f, m = a.min_p ? a.min_p[r] : 0.0f;
    const int k = a.top_k ? a.top_k[r] : 0;
    const float u = a.u[r];
    auto answer = [&](uint32_t token, float prob, uint32_t kept) {
        if (threadIdx.x) return;
        a.token[r] = (int32_t)token;
        if (a.prob) a.prob[r] = prob;
        if (a.kept) a.kept[r] = (int32_t)kept;
    };

    float mine = attn::NEG_INF;
    row.each([&](float l, int) { mine = fmaxf(mine, l); });
    float top = over_wave(mine, [](float x, float y) { return fmaxf(x, y); });
    if (lane == 0) s.tmp32[wave] = __float_as_uint(top);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, __uint_as_float(s.tmp32[w]));
    __syncthreads();
    if (!(top > attn::NEG_INF)) return answer(~0u, 0.0f, 0);
    if (!(T > 0.0f) || k == 1 || p <= 0.0f) {  // the first of the largest
        uint32_t first = ~0u;
        row.each([&](float l, int i) {
            if (l == top) first = min(first, (uint32_t)i);
        });
        first = over_wave(first, [](uint32_t x, uint32_t y) { return min(x, y); });
        if (lane == 0) s.tmp32[wave] = first;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) first = min(first, s.tmp32[w]);
        return answer(first, 1.0f, 1);
    }
    const Scale sc = {top, PER_UNIT / T, 1.44269504088896340736 / (double)T};

    // the list: the first tokens of the order, enough of them for every question
    int n = LIST + 1;       // in the list; more than LIST: not collected
    bool whole = false;     // the list holds every token, or `total` is the weight of all
    u64 total = 0;
    if (k > 0 && k <= SMALL_K) {
        // the k-th largest of the threads' maxima, to 16 bits of its key
        uint32_t bound = 0;
        uint32_t want = (uint32_t)k;
        const uint32_t key = key_of(mine);
#pragma unroll 1
        for (int shift = 24; shift >= 16; shift -= 8) {
            for (int i = threadIdx.x; i < 256; i += THREADS) s.digits.count[i] = 0;
            __syncthreads();
            if (shift == 24 || key >> 24 == bound >> 24) atomicAdd(&s.digits.count[key >> shift & 255], 1u);
            __syncthreads();
            if (wave == 0) {
                uint32_t c[4], sum = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    c[i] = s.digits.count[lane * 4 + i];
                    sum += c[i];
                }
                uint32_t upto = sum;
#pragma unroll
                for (int o = 1; o < SAE_WAVE; o <<= 1) {
                    const uint32_t x = __shfl_up(upto, o);
                    if (lane >= o) upto += x;
                }
                uint32_t before = upto - sum;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (before < want && before + c[i] >= want) {
                        s.found = lane * 4 + i;
                        s.n = want - before;
                    }
                    before += c[i];
                }
            }
            __syncthreads();
            bound |= s.found << shift;
            want = s.n;
            __syncthreads();
        }
        bound |= 0xFFFFu;  // keys up to it
        if (threadIdx.x == 0) s.n = 0;
        __syncthreads();
        row.each([&](float l, int i) {
            const uint32_t x = key_of(l);
            if (l > attn::NEG_INF && x <= bound) {
                const uint32_t at = atomicAdd(&s.n, 1u);
                if (at < LIST) s.list[at] = (u64)x << 32 | (uint32_t)i;
            }
        });
        __syncthreads();
        n = uniform((int)s.n);
    }
    u64 kth = 0;  // tokens that top-k leaves
    if (n > LIST) {
        clear(s.bins);
        __syncthreads();
        uint32_t light = 0;  // tokens of the last bin
        row.each([&](float l, int) {
            if (!(l > attn::NEG_INF)) return;
            const int b = sc.bin(l);
            if (b == BINS - 1) {
                ++light;
                return;
            }
            atomicAdd(&s.bins.count[b], 1u);
            atomicAdd(&s.bins.mass[b], sc.weight(l));
        });
        light = over_wave(light, [](uint32_t x, uint32_t y) { return x + y; });
        if (lane == 0 && light) atomicAdd(&s.bins.count[BINS - 1], light);
        __syncthreads();
        accumulate(s, s.bins);
        const uint32_t all = s.bins.count[BINS - 1];
        total = s.bins.mass[BINS - 1];
        kth = k > 0 && (uint32_t)k < all ? (uint32_t)k : all;
        int last = first_bin(s, s.bins, [&](uint32_t c, u64) { return c >= kth; });
        whole = kth == all;
        // (top-p of what top-k leaves: its weight has to be known first)
        if (p < 1.0f && whole) {
            const u64 most = share(p, total, true);
            last = min(last, first_bin(s, s.bins, [&](uint32_t, u64 mass) { return mass >= most; }));
        }
        if (m > 0.0f && (whole || !(p < 1.0f))) {
            const float x = -__builtin_logf(fminf(m, 1.0f)) * PER_UNIT + 2.0f;
            if (x < (float)last) last = (int)x;
        }
        n = (int)s.bins.count[last];
        if (n <= LIST) {
            if (threadIdx.x == 0) s.n = 0;
            __syncthreads();
            row.each([&](float l, int i) {
                if (l > attn::NEG_INF && sc.bin(l) <= last) s.list[min(atomicAdd(&s.n, 1u), (uint32_t)LIST - 1)] = (u64)key_of(l) << 32 | (uint32_t)i;
            });
            __syncthreads();
        }
    }
    if (n <= LIST) {
        sort_and_sum(s, sc, n, 0);
        int keep = k > 0 ? min(k, n) : n;
        const u64 of = whole ? total : uniform64(s.sums[keep - 1]);
        if (p < 1.0f) {
            const u64 target = share(p, of, true);
            keep = min(keep, first_sum(s, n, [&](u64 sum) { return sum >= target; }) + 1);
        }
        if (m > 0.0f) {
            const double least = (double)m * ONE;
            __syncthreads();
            if (threadIdx.x == 0) s.found = keep;
            __syncthreads();
            for (int i = threadIdx.x; i < keep; i += THREADS)
                if ((double)(s.sums[i] - (i ? s.sums[i - 1] : 0)) < least) atomicMin(&s.found, (uint32_t)i);
            __syncthreads();
            keep = max(1, uniform((int)s.found));
        }
        const u64 sum = uniform64(s.sums[keep - 1]);
        const u64 target = u > 0.0f ? min(share(fminf(u, 1.0f), sum, false), sum - 1) : 0;
        const int at = first_sum(s, keep, [&](u64 x) { return x > target; });
        const u64 w = s.sums[at] - (at ? s.sums[at - 1] : 0);
        return answer((uint32_t)s.list[at], (float)((double)w / (double)sum), keep);
    }
    // too many for the list: each question by itself
    Head h = {kth, total, 0, 0};
#pragma unroll 1
    for (int question = 0;; ++question) {  // top-k, top-p, min-p, the token
        if ((question == 0 && whole) || (question == 1 && !(p < 1.0f)) || (question == 2 && !(m > 0.0f))) continue;
        if (question != 2) {
            const u64 target = question == 0 ? kth : question == 1 ? max(share(p, h.mass, true), 1ull)
                               : u > 0.0f ? min(share(fminf(u, 1.0f), h.mass, false), h.mass - 1) + 1 : 1;
            const Head found = locate(s, row, sc, question == 0, target, question == 3);
            if (question == 3) return answer(found.index, (float)((double)found.last / (double)h.mass), (uint32_t)h.n);
            h = found;
            continue;
        }
        const double least = (double)m * ONE;
        uint32_t c = 0;
        u64 mass = 0;
        row.each([&](float l, int) {
            if (!(l > attn::NEG_INF)) return;
            const u64 w = sc.weight(l);
            if ((double)w >= least) {
                ++c;
                mass += w;
            }
        });
        u64 c_all, m_all;
        scan<NW>((u64)c, c_all, s.tmp);
        __syncthreads();
        scan<NW>(mass, m_all, s.tmp);
        if (c_all == 0) {
            c_all = 1;
            m_all = (u64)ONE;
        }
        if (c_all < h.n) h = {c_all, m_all, 0, 0};
    }
}

}  // namespace

size_t sample_work_bytes(int, int) { return 16; }

hipError_t launch_sample(int rows, int vocab, int dtype, const SampleArgs &x, hipStream_t s)
{
    const Args a = {x.logits, x.stride, x.settings.temperature, x.settings.top_p, x.settings.min_p, x.u, x.settings.top_k,
                    x.token, x.kept, x.prob, vocab};
    if (dtype == SAE_KV_BF16) hipLaunchKernelGGL((k_sample<SAE_KV_BF16>), dim3(rows), dim3(THREADS), 0, s, a);
    else if (dtype == SAE_KV_F16) hipLaunchKernelGGL((k_sample<SAE_KV_F16>), dim3(rows), dim3(THREADS), 0, s, a);
    else hipLaunchKernelGGL((k_sample<SAE_ROWS_F32>), dim3(rows), dim3(THREADS), 0, s, a);
    return hipGetLastError();
}
