// Attention of one new token per sequence over the paged key-value cache.
//
// Per sequence and key-value head, with the G query heads that share it as the
// columns of a 16-wide matrix (G of them used; more than 16 take several tiles):
//   S^T = K Q^T (32 keys x 16 heads a step), P = exp(S - m), O^T += V^T P^T
// on v_mfma_f32_16x16x32, m and the sum of P running (one pass over the keys).
// The time is that of reading the cache once: the matrix units are used because
// they take every cached byte from the register it was loaded into, for 16 heads
// at the price of one.
//
// Everything stays in registers: lane (n = lane % 16, g = lane / 16) holds the
// scores of head n for 8 of the 32 keys, and the same 8 keys are what lane
// group g supplies of V^T and P^T to the second product, because the 32 rows of
// K are taken in the order that makes it so (below) and because the sum over
// keys may be taken in any order that both operands share.  So neither P nor
// the output passes through LDS or other lanes; the running maximum needs two
// swaps across lane groups a step.
//   first product, tile u = 0, 1: row 4 g' + i is token 8 u + 4 (g' % 2) + i of
//     page g' / 2 of the step's two pages
//   second product: k = 8 g + j is, for j < 4, token 4 (g % 2) + j of page g / 2,
//     for j >= 4 token 8 + 4 (g % 2) + j - 4: the 8 tokens of a value page's
//     16-byte piece.
//
// Bound by memory: 256 sequences of 512..2,048 tokens (8 heads of 128, bf16; 1.35 GB,
// 1.36 GB fetched) 238 us, 5.6 TB/s; 131,072 tokens of the 8-bit cache 53.7 us and 4.7
// for the join; of the matrix units' time 24 products of 16 cycles go with the 16 KB of a
// step, a twelfth of what a compute unit could feed from memory.  So weights go into
// the second product as two 16-bit numbers, f16 ones 2^15 times as large (weights
// down to 2^-40 of a head's largest count): its error is then that of the output's
// rounding alone.  Smallest calls are round trips: 7 us, and 3.5 for a join.
//
// Work is divided evenly whatever the lengths: all sequences' steps lie one
// after the other, and workgroup x takes steps x per .. (x + 1) per - 1 of its
// head, found from the lengths alone (a scan in every workgroup: the host knows
// no lengths, and a captured call keeps fitting as they grow).  A sequence that
// lies in one workgroup is finished there; the parts of others go to the
// workspace and k_decode_join adds them.  A workgroup has at most two such
// parts: its first sequence's end and its last one's beginning.
#include "attn_tile.h"

namespace {

using namespace attn;

constexpr int NW = 4, THREADS = NW * SAE_WAVE;
constexpr int STEP = 32;       // keys a wave takes at a time: two pages
constexpr int COLS = 16;       // query heads of a tile
constexpr int MIN_STEPS = NW;  // steps of a workgroup at least (where there are as many)
// Steps that a sequence costs beside its own (37 sequences of 1..36,000 tokens: 0: 46.6
// us, 4: 39.5, 8: 35.4, 16: 36.7; 256 of 512..2,048: 243 us up to 12, 248 at 16).
constexpr int EXTRA = 8;
// Bytes of keys and values up to which a sequence is left to one workgroup per head
// (from the table's width: a second launch and the scan cost more than one compute
// unit takes for them).  Drawn batches of short sequences, geometric means of 12 calls,
// three draws: never 17.4 / 16.2 / 20.0 us, up to 192 KB 13.3 / 13.3 / 15.2, up to 400
// KB 13.3 / 12.7 / 15.5, up to 1,000 KB 13.4 / 12.7 / 15.2.
constexpr int64_t SINGLE = 384 << 10;
// Workgroups of a call, about: two per compute unit (768: 247 us for the batch above, 65
// for the long one; 1,024: 250 and 65).
constexpr int GROUPS = 512;
template <bool F16>
constexpr float BIAS = F16 ? 15.0f : 0.0f;  // of the weights' reference: weights up to 2^BIAS

// Two values rounded to the 16-bit type, and what the rounding left, rounded too.
template <bool F16>
__device__ __forceinline__ void split2(float a, float b, uint32_t &hi, uint32_t &lo)
{
    hi = pack2<F16>(a, b);
    lo = pack2<F16>(a - low<F16>(hi), b - high<F16>(hi));
}

__device__ __forceinline__ float sum_groups(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// First key and number of steps of a sequence of n tokens (one step, which
// sees nothing, where there is no key: its workgroup writes the zeros).
__device__ __forceinline__ int first_key(int n, int window) { return window > 0 ? max(n - window, 0) : 0; }
__device__ __forceinline__ int steps_of(int n, int window)
{
    return n <= 0 ? 1 : (n + STEP - 1) / STEP - first_key(n, window) / STEP;
}

// What a sequence costs its workgroup: its steps and, behind them, as much as EXTRA
// steps take for its start and end (round trips for its table and first keys, the
// waves' parts joined).
__device__ __forceinline__ int cost_of(int n, int window) { return steps_of(n, window) + EXTRA; }

// Steps per workgroup, for `total` steps over `groups` workgroups.
__device__ __forceinline__ long long steps_per(long long total, int groups)
{
    const long long p = (total + groups - 1) / groups;
    return p < MIN_STEPS ? MIN_STEPS : p;
}

// Where workgroup x of a head starts: its first sequence and the step in it.
struct Start {
    long long per, begin, end;  // steps begin .. end - 1 of all
    int seq, len;               // that sequence and its length
    long long seq_at;           // number of its first step
};

__device__ __forceinline__ Start find_start(const KvDev &c, int window, int x, int groups)
{
    __shared__ long long tmp[NW];
    __shared__ uint32_t tmp32[NW];
    __shared__ long long found_at;
    __shared__ int found_seq, found_len;
    const int n = c.n_seq, chunk = (n + THREADS - 1) / THREADS;
    const int r0 = min((int)threadIdx.x * chunk, n), r1 = min(r0 + chunk, n);
    Start s;
    long long total, at, sum = 0;
    int len = 0;
    if (chunk == 1) {  // 32 bits are enough: 256 sequences of 2^23 steps at most
        if (r0 < n) {
            len = kv::seq_len(c, r0);
            sum = cost_of(len, window);
        }
        uint32_t t32;
        at = scan<NW>((uint32_t)sum, t32, tmp32);
        total = t32;
    } else {
        for (int r = r0; r < r1; ++r) sum += cost_of(kv::seq_len(c, r), window);
        at = scan<NW>(sum, total, tmp);
    }
    s.per = steps_per(total, groups);
    s.begin = x * s.per;
    s.end = min(s.begin + s.per, total);
    if (s.begin < total && at <= s.begin && s.begin < at + sum) {  // one thread
        int r = r0;
        if (chunk > 1)
            for (;; ++r) {
                len = kv::seq_len(c, r);
                const int k = cost_of(len, window);
                if (s.begin < at + k) break;
                at += k;
            }
        found_seq = r;
        found_len = len;
        found_at = at;
    }
    __syncthreads();
    const bool any = s.begin < total;
    s.seq = __builtin_amdgcn_readfirstlane(any ? found_seq : n);
    s.len = __builtin_amdgcn_readfirstlane(any ? found_len : 0);
    s.seq_at = any ? found_at : total;
    return s;
}

// Workspace: descriptions of split sequences, by sequence where there are no more
// of them than workgroups (the join then has a workgroup for each), else by the
// workgroup x in which the sequence begins (one at most continues past it); then per (x, head tile, slot) 16 maxima, 16 sums and
// 16 rows of unnormalised outputs.
struct Part {
    int seq, first, count;  // its parts: workgroups first .. first + count - 1; count < 2: none to join
    int pad;
};
__host__ __device__ constexpr size_t part_floats(int dim) { return (size_t)COLS * (dim + 2); }
__host__ __device__ constexpr size_t meta_bytes(int groups) { return ((size_t)groups * sizeof(Part) + 15) / 16 * 16; }

struct Shape {
    int groups, tiles, per_kv;  // workgroups per head tile; head tiles in all; head tiles of a key-value head
    int by_seq;                 // descriptions go by sequence
    int single;                 // one workgroup per sequence and head tile: none is split
};

// One step's keys and values of a lane, as loaded.
template <int TYPE, int D>
struct Frag {
    static constexpr int NK = TYPE == SAE_KV_FP8 ? D / 64 : D / 32;  // pieces of a row tile
    static constexpr int NV = TYPE == SAE_KV_FP8 ? D / 32 : D / 16;
    u32x4 k[2][NK], v[NV];
    uint32_t ks[2], vs[2];  // scale bytes of the lane's 8 keys
};

template <int TYPE, int D>
__global__ void __launch_bounds__(THREADS, D == 256 ? 1 : 2) k_decode(KvDev c, AttnArgs a, Shape sh)
{
    constexpr bool FP8 = TYPE == SAE_KV_FP8, F16 = is_f16(TYPE);
    constexpr int E = FP8 ? 1 : 2, PAGE = SAE_KV_BLOCK * D * E;
    constexpr int NO = D / 16, NQ = D / 32;
    typedef Frag<TYPE, D> F;
    constexpr int OROW = D + 4;  // LDS row of an output, padded against conflicts
    __shared__ float ox[NW][COLS][OROW];
    __shared__ float mx[NW][COLS], lx[NW][COLS];

    const int x = blockIdx.x, tile = blockIdx.y;
    const int kvhead = tile / sh.per_kv, G = a.heads / c.kvh;
    const int head0 = kvhead * G + tile % sh.per_kv * COLS;
    const int cols = min(COLS, G - tile % sh.per_kv * COLS);
    const int lane = (int)__lane_id(), wave = threadIdx.x / SAE_WAVE;
    const int n = lane & 15, g = lane >> 4;
    Start st;
    if (sh.single) {
        st.seq = x;
        st.len = kv::seq_len(c, x);
        st.seq_at = st.begin = 0;
        st.per = st.end = 1ll << 40;
    } else {
        st = find_start(c, a.window, x, sh.groups);
    }
    Part *meta = reinterpret_cast<Part *>(a.work);
    float *parts = reinterpret_cast<float *>(static_cast<char *>(a.work) + meta_bytes(sh.groups));
    Part mine = {0, 0, 0, 0};
    const float sl = a.scale * LOG2E;
    // the lane's place in a page (bytes)
    const int koff = g * 256 + (lane & 7) * 16, voff = (lane & 15) * 32 + (g & 1) * 16;
    const bool kpage = lane & 8, vpage = lane & 32;

    long long at = st.begin, seq_at = st.seq_at;
    for (int r = st.seq, len = st.len, next = 0; at < st.end; ++r, len = kv::checked_len(c, next)) {
        const int total = steps_of(len, a.window);
        if (!sh.single) next = c.len[min(r + 1, c.n_seq - 1)];  // on its way while this sequence is taken
        const int lo = first_key(len, a.window);
        const int s0 = (int)(at - seq_at), s1 = (int)min((long long)total, st.end - seq_at);
        const long long after = seq_at + total + EXTRA;
        if (s0 >= total) {  // uniform: the workgroup before had its last step
            at = seq_at = after;
            continue;
        }
        const int step0 = lo / STEP;  // in steps of the whole sequence
        const int64_t base = kv::seq_base(c, r);
        u32x4 q[NQ];
        {
            const char *qr = static_cast<const char *>(a.q) + ((int64_t)r * a.q_stride + (int64_t)(head0 + n) * D) * 2;
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                // 8-bit keys come 16 dimensions a piece: piece i / 2 of lane group g, its half i % 2
                const int d = FP8 ? i / 2 * 64 + g * 16 + i % 2 * 8 : i * 32 + g * 8;
                q[i] = u32x4{0, 0, 0, 0};
                if (n < cols) q[i] = *reinterpret_cast<const u32x4 *>(qr + d * 2);
            }
        }
        f32x4 o[NO];
#pragma unroll
        for (int i = 0; i < NO; ++i) o[i] = f32x4{0, 0, 0, 0};
        float m = NEG_INF, l = 0.0f;  // m: the reference of weights

        // table entries of the wave's next 32 steps: lane 2 j + u has page u of step j
        int ids = -1, ids_from = -1;
        const int count = (s1 - s0 - wave + NW - 1) / NW;  // this wave's steps: s0 + wave + NW j
        auto fetch = [&](F &f, int j, bool &v0, bool &v1) {
            if (j >= count) return;
            if (ids_from < 0 || j >= ids_from + 32) {  // uniform
                ids_from = j;
                const int page = 2 * (step0 + s0 + wave + NW * (j + (lane >> 1))) + (lane & 1);
                // (the first load need not wait for the length)
                ids = page < c.max_blocks ? c.ids[(int64_t)r * c.max_blocks + page] : -1;
                if (j + (lane >> 1) >= count || page * SAE_KV_BLOCK >= len) ids = -1;
                if (ids >= c.bpi) kv::report(c);
                if (base < 0 || ids >= c.bpi) ids = -1;
            }
            const int i0 = __builtin_amdgcn_readlane(ids, 2 * (j - ids_from));
            const int i1 = __builtin_amdgcn_readlane(ids, 2 * (j - ids_from) + 1);
            v0 = i0 >= 0;
            v1 = i1 >= 0;
            // a page that is not there is read as block 0, and masked
            const int64_t b0 = v0 ? base + i0 : 0, b1 = v1 ? base + i1 : 0;
            const int64_t a0 = b0 * c.block_bytes + (int64_t)kvhead * PAGE, a1 = b1 * c.block_bytes + (int64_t)kvhead * PAGE;
            const char *kp = c.k + (kpage ? a1 : a0) + koff, *vp = c.v + (vpage ? a1 : a0) + voff;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < F::NK; ++i) f.k[u][i] = *reinterpret_cast<const u32x4 *>(kp + i * 1024 + u * 128);
#pragma unroll
            for (int i = 0; i < F::NV; ++i) f.v[i] = *reinterpret_cast<const u32x4 *>(vp + i * 512);
            if constexpr (FP8) {
                const int64_t s = (vpage ? b1 : b0) * c.scale_stride + kvhead * SAE_KV_BLOCK + (g & 1) * 4;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    f.ks[u] = *reinterpret_cast<const uint32_t *>(c.ks + s + u * 8);
                    f.vs[u] = *reinterpret_cast<const uint32_t *>(c.vs + s + u * 8);
                }
            }
        };
        auto compute = [&](F &f, int j, bool v0, bool v1) {
            const int t0 = (step0 + s0 + wave + NW * j) * STEP;
            f32x4 s[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                s[u] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < F::NK; ++i) {
                    if constexpr (FP8) {
                        s[u] = mfma16<F16>(widen8(f.k[u][i][0], f.k[u][i][1], 1.0f), q[2 * i], s[u]);
                        s[u] = mfma16<F16>(widen8(f.k[u][i][2], f.k[u][i][3], 1.0f), q[2 * i + 1], s[u]);
                    } else {
                        s[u] = mfma16<F16>(f.k[u][i], q[i], s[u]);
                    }
                }
            }
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = s[e / 4][e % 4] * sl;
                if constexpr (FP8) w[e] *= scale_of(f.ks[e / 4], e % 4);
            }
            if (!v0 || !v1 || t0 < lo || t0 + STEP > len) {  // uniform: some key of the step is not seen
                asm volatile("");  // a branch: not worth taking on every step
                // lo <= key < len of a page that is there: key - lo, without sign, is below seen
                const uint32_t seen = (vpage ? v1 : v0) ? (uint32_t)(len - lo) : 0u;
                const uint32_t rel = (uint32_t)(t0 + (g >> 1) * SAE_KV_BLOCK + (g & 1) * 4 - lo);
                // a value that is not seen may be NaN: it becomes 0, and its scale byte too
                uint32_t keep[4] = {0, 0, 0, 0};  // of the values: two 16-bit ones a word, or four bytes (two words)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool there = rel + (uint32_t)(e / 4 * 8 + e % 4) < seen;
                    if (!there) w[e] = NEG_INF;
                    if constexpr (FP8) keep[e / 4] |= there ? 0xFFu << (8 * (e % 4)) : 0u;
                    else keep[e / 2] |= there ? 0xFFFFu << (16 * (e % 2)) : 0u;
                }
#pragma unroll
                for (int i = 0; i < F::NV; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) f.v[i][k] &= keep[FP8 ? k & 1 : k];
                if constexpr (FP8) {
                    f.vs[0] &= keep[0];
                    f.vs[1] &= keep[1];
                }
            }
            float top = w[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) top = fmaxf(top, w[e]);
            top = reference<F16>(max_groups(top), BIAS<F16>);
            if (__any(top > m)) {  // a head's maximum grew: what is summed so far shrinks
                const float mn = fmaxf(m, top);
                const float f0 = mn == NEG_INF ? 0.0f : exp2_(m - mn);
                m = mn;
                l *= f0;
#pragma unroll
                for (int i = 0; i < NO; ++i) o[i] *= f0;
            }
            const float mu = m == NEG_INF ? 0.0f : m;  // nothing seen yet
            u32x4 hi, lo_;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = exp2_(w[e] - mu);
                l += w[e];
                if constexpr (FP8) w[e] *= scale_of(f.vs[e / 4], e % 4);
            }
            // the weights as two 16-bit numbers each: the product with the values
            // costs twice the (idle) matrix units and keeps 16 bits or more of them (f16: 22, or
            // what lies above 2^-39 of the largest)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t h_, l_;
                split2<F16>(w[2 * e], w[2 * e + 1], h_, l_);
                hi[e] = h_;
                lo_[e] = l_;
            }
#pragma unroll
            for (int i = 0; i < NO; ++i) {
                const u32x4 v = FP8 ? widen8(f.v[i / 2][i % 2 * 2], f.v[i / 2][i % 2 * 2 + 1], 1.0f) : f.v[FP8 ? 0 : i];
                o[i] = mfma16<F16>(v, hi, o[i]);
                o[i] = mfma16<F16>(v, lo_, o[i]);
            }
        };
        // the next step's loads are in flight while one is computed
        F f0, f1;
        bool va0 = false, va1 = false, vb0 = false, vb1 = false;
        fetch(f0, 0, va0, va1);
        for (int j = 0; j < count; j += 2) {
            fetch(f1, j + 1, vb0, vb1);
            compute(f0, j, va0, va1);
            if (j + 1 < count) {
                fetch(f0, j + 2, va0, va1);
                compute(f1, j + 1, vb0, vb1);
            }
        }

        // the waves' parts: common maximum, sums, outputs
        l = sum_groups(l);
        __syncthreads();  // the last sequence's sums have been read
        if (g == 0) {
            mx[wave][n] = m;
            lx[wave][n] = l;
        }
#pragma unroll
        for (int i = 0; i < NO; ++i) *reinterpret_cast<f32x4 *>(&ox[wave][n][i * 16 + g * 4]) = o[i];
        __syncthreads();
        const bool whole = s0 == 0 && s1 == total;
        const size_t slot = ((size_t)x * sh.tiles + tile) * 2 + (s0 == 0 ? 1 : 0);
        float *pm = parts + slot * part_floats(D), *po = pm + 2 * COLS;
        for (int i = threadIdx.x; i < cols * (D / 4); i += THREADS) {
            const int h = i / (D / 4), d = i % (D / 4) * 4;
            float top = NEG_INF;
#pragma unroll
            for (int w = 0; w < NW; ++w) top = fmaxf(top, mx[w][h]);
            f32x4 sum = {0, 0, 0, 0};
            float z = 0.0f;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float f = mx[w][h] == NEG_INF ? 0.0f : exp2_(mx[w][h] - top);
                z += lx[w][h] * f;
                sum += *reinterpret_cast<const f32x4 *>(&ox[w][h][d]) * f;
            }
            if (whole) {
                const float inv = z == 0.0f ? 0.0f : 1.0f / z;  // no key, or every score -inf
                const int64_t to = (int64_t)r * a.out_stride + (int64_t)(head0 + h) * D + d;
                *reinterpret_cast<u32x2 *>(static_cast<char *>(a.out) + to * 2) =
                    u32x2{pack2<F16>(sum[0] * inv, sum[1] * inv), pack2<F16>(sum[2] * inv, sum[3] * inv)};
                if (a.lse && d == 0)
                    a.lse[(int64_t)r * a.heads + head0 + h] = z == 0.0f ? NEG_INF : (top + log2_(z)) * LN2;
            } else {
                *reinterpret_cast<f32x4 *>(po + h * D + d) = sum;
                if (d == 0) {
                    pm[h] = top;
                    pm[COLS + h] = z;
                }
            }
        }
        if (sh.single) return;
        if (s0 == 0) {
            const Part p = {r, x, (int)((seq_at + total - 1) / st.per) - x + 1, 0};
            if (sh.by_seq && tile == 0 && threadIdx.x == 0) meta[r] = p;
            if (p.count > 1) mine = p;
        }
        at = seq_at = after;
    }
    if (!sh.by_seq && tile == 0 && threadIdx.x == 0) meta[x] = mine;
}

// Joins a split sequence's parts: one workgroup per (description, query head), its
// threads in JR rows of D / 4, row i taking parts i, i + JR, ..., UN of them at once.
template <int TYPE, int D>
__global__ void __launch_bounds__(THREADS) k_decode_join(KvDev c, AttnArgs a, Shape sh)
{
    constexpr int LD = D / 4, JR = THREADS / LD, UN = 4;
    __shared__ float mz[JR], zz[JR];
    __shared__ f32x4 oz[JR][LD];
    const int head = blockIdx.y;
    const Part p = reinterpret_cast<const Part *>(a.work)[blockIdx.x];
    if (p.count < 2) return;
    const float *parts = reinterpret_cast<const float *>(static_cast<const char *>(a.work) + meta_bytes(sh.groups));
    const int G = a.heads / c.kvh, u = head % G;
    const int tile = head / G * sh.per_kv + u / COLS, h = u % COLS;
    const int row = threadIdx.x / LD, d = threadIdx.x % LD;
    float m = NEG_INF, z = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    for (int i = row; i < p.count; i += JR * UN) {
        float mi[UN], zi[UN];
        f32x4 oi[UN];
#pragma unroll
        for (int k = 0; k < UN; ++k) {
            const int j = min(i + k * JR, p.count - 1);  // past the end: weighs nothing below
            const float *pm = parts + (((size_t)(p.first + j) * sh.tiles + tile) * 2 + (j == 0 ? 1 : 0)) * part_floats(D);
            mi[k] = pm[h];
            zi[k] = pm[COLS + h];
            oi[k] = *reinterpret_cast<const f32x4 *>(pm + 2 * COLS + h * D + d * 4);
        }
        float top = m;
#pragma unroll
        for (int k = 0; k < UN; ++k)
            if (i + k * JR < p.count) top = fmaxf(top, mi[k]);
        const float mu = top == NEG_INF ? 0.0f : top, f = exp2_(m - mu);
        o *= f;
        z *= f;
#pragma unroll
        for (int k = 0; k < UN; ++k)
            if (i + k * JR < p.count) {
                const float fk = exp2_(mi[k] - mu);
                o += oi[k] * fk;
                z += zi[k] * fk;
            }
        m = top;
    }
    if (d == 0) {
        mz[row] = m;
        zz[row] = z;
    }
    oz[row][d] = o;
    __syncthreads();
    if (row != 0) return;
    float top = NEG_INF;
#pragma unroll
    for (int i = 0; i < JR; ++i) top = fmaxf(top, mz[i]);
    const float mu = top == NEG_INF ? 0.0f : top;
    z = 0.0f;
    o = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < JR; ++i) {
        const float f = exp2_(mz[i] - mu);
        z += zz[i] * f;
        o += oz[i][d] * f;
    }
    const float inv = z == 0.0f ? 0.0f : 1.0f / z;
    const int64_t to = (int64_t)p.seq * a.out_stride + (int64_t)head * D + d * 4;
    *reinterpret_cast<u32x2 *>(static_cast<char *>(a.out) + to * 2) =
        u32x2{pack2<is_f16(TYPE)>(o[0] * inv, o[1] * inv), pack2<is_f16(TYPE)>(o[2] * inv, o[3] * inv)};
    if (a.lse && d == 0)
        a.lse[(int64_t)p.seq * a.heads + head] = z == 0.0f ? NEG_INF : (top + log2_(z)) * LN2;
}

Shape shape_of(int heads, int kvh, int n_seq, int64_t longest = 1ll << 40)
{
    Shape s;
    s.per_kv = (heads / kvh + COLS - 1) / COLS;
    s.tiles = kvh * s.per_kv;
    s.groups = GROUPS / s.tiles > 1 ? GROUPS / s.tiles : 1;
    s.by_seq = n_seq <= s.groups;
    s.single = longest <= SINGLE;
    return s;
}

template <int TYPE, int D>
hipError_t launch(const KvDev &c, const AttnArgs &a, hipStream_t s)
{
    // bytes of the longest sequence that the table holds (or the window lets be seen), per head
    int64_t longest = (int64_t)c.max_blocks * SAE_KV_BLOCK;
    if (a.window > 0 && longest > a.window) longest = a.window;
    const Shape sh = shape_of(a.heads, c.kvh, c.n_seq, longest * 2 * D * (TYPE == SAE_KV_FP8 ? 1 : 2));
    hipLaunchKernelGGL((k_decode<TYPE, D>), dim3(sh.single ? c.n_seq : sh.groups, sh.tiles), dim3(THREADS), 0, s, c, a, sh);
    hipError_t e = hipGetLastError();
    // one workgroup per head or per sequence: none is split
    if (e != hipSuccess || sh.groups == 1 || sh.single) return e;
    hipLaunchKernelGGL((k_decode_join<TYPE, D>), dim3(sh.by_seq ? c.n_seq : sh.groups, a.heads), dim3(THREADS),
                       0, s, c, a, sh);
    return hipGetLastError();
}

template <int TYPE>
hipError_t launch_dim(const KvDev &c, const AttnArgs &a, int dim, hipStream_t s)
{
    return dim == 64 ? launch<TYPE, 64>(c, a, s) : dim == 128 ? launch<TYPE, 128>(c, a, s) : launch<TYPE, 256>(c, a, s);
}

}  // namespace

size_t decode_work_bytes(int heads, int kvh, int dim)
{
    const Shape s = shape_of(heads, kvh, 0);
    return meta_bytes(s.groups) + (size_t)s.groups * s.tiles * 2 * part_floats(dim) * sizeof(float);
}

hipError_t launch_decode(const KvDev &c, const AttnArgs &a, int type, int dim, hipStream_t s)
{
    if (type == SAE_KV_BF16) return launch_dim<SAE_KV_BF16>(c, a, dim, s);
    if (type == SAE_KV_F16) return launch_dim<SAE_KV_F16>(c, a, dim, s);
    return launch_dim<SAE_KV_FP8>(c, a, dim, s);
}
