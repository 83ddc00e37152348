// Causal attention of sequences' new tokens over the paged key-value cache.
//
// The query rows of a sequence and key-value head are its new tokens times the
// G query heads that share the head, row = token * G + head: keys and values are
// read once for all of them.  A workgroup takes a tile of 32 NW rows, a wave 32
// of them, over 64 keys (4 pages) a step, with the scores transposed:
//   S^T = K Q^T (64 keys x 32 rows), P = exp(S - m), O^T += V^T P^T
// on v_mfma_f32_32x32x16.  Keys and values of a step are staged in LDS, in the
// cache's own page layout, double-buffered, the next step's loads in flight in
// registers; an 8-bit cache is widened to bf16 (times its scale) on the way, once
// for all waves.  Queries, scores, weights and outputs never leave registers:
// lane (n = lane % 32, h = lane / 32) holds all of row n's state (the other half
// of its keys and dimensions in lane n ^ 32), and the 16 scores a lane holds of 32
// keys are, rounded, the operand of the second product as they stand:
//   registers 8 u .. 8 u + 7 are tokens 4 h .. 4 h + 3 and 8 + 4 h .. of page u,
// which is the 16-byte piece h of a value page's dimension.
//
// The running maximum is followed loosely: outputs are rescaled only when some
// row's maximum grew by more than 2^8, so weights are at most 2^8 (sums are fp32).
//
// Where tiles are few, each one's keys are split over several workgroups, whose
// unnormalised outputs k_prefill_join adds in order.
#include "attn_tile.h"

namespace {

using namespace attn;

constexpr int ROWS = 32;   // rows of a wave
constexpr int KEYS = 64;   // keys of a step
constexpr int PAGES = KEYS / SAE_KV_BLOCK;
constexpr int MIN_SPLIT = 4;     // steps of a split at least
constexpr int GROUPS = 512;      // workgroups wanted: two per compute unit
constexpr float SLACK = 8.0f;    // of the running maximum, in powers of two

// Orders LDS only: loads from memory stay in flight across it.
__device__ __forceinline__ void barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

struct Plan {
    int tiles;   // row tiles of a head (an upper bound), `splits` workgroups each
    int splits;
};

// The rows of a workgroup and the keys they see.
struct Tile {
    int seq, first;        // first row of the sequence in the call's arrays
    int tokens;            // its new tokens
    int64_t row0;          // first row of the tile: token0 * G + head0
    int token0, head0;
    int rows;              // rows of the tile that there are
    int pos0;              // position of its first new token (may be negative)
    int len;
    int step0, steps;      // steps of KEYS keys the tile sees: step0 .. step0 + steps - 1
    int parts;             // workgroups they are divided over
    bool none;
};

__device__ __forceinline__ Tile tile_of(const KvDev &c, const AttnArgs &a, int64_t tile, int rows, int splits)
{
    Tile t;
    const int G = a.heads / c.kvh;
    int64_t sub;
    if (!c.qs) {
        const int of_seq = (G + rows - 1) / rows;
        t.seq = (int)(tile / of_seq);
        sub = tile % of_seq;
    } else {
        // f(r) = q_start[r] G / rows + r: at least the tiles before sequence r
        int lo = 0, n = c.n_seq;
        while (n > 1) {
            const int step = (n + SAE_WAVE - 1) / SAE_WAVE, r = lo + (int)__lane_id() * step;
            const bool below = r < lo + n && (int64_t)c.qs[r] * G / rows + r <= tile;
            const uint64_t m = __ballot(below);
            const int last = m ? 63 - __clzll((long long)m) : 0, end = lo + n;
            lo += last * step;
            n = min(step, end - lo);
        }
        t.seq = __builtin_amdgcn_readfirstlane(lo);
        sub = tile - ((int64_t)c.qs[t.seq] * G / rows + t.seq);
    }
    kv::seq_rows(c, t.seq, t.first, t.tokens);
    t.row0 = sub * rows;
    t.none = sub < 0 || t.row0 >= (int64_t)t.tokens * G;
    t.len = kv::seq_len(c, t.seq);
    t.pos0 = t.len - t.tokens;
    t.step0 = t.steps = 0;
    t.parts = 1;
    if (t.none) return t;
    const int64_t end = min(t.row0 + rows, (int64_t)t.tokens * G);
    t.rows = (int)(end - t.row0);
    t.token0 = (int)(t.row0 / G);
    t.head0 = (int)(t.row0 % G);
    const int p0 = t.pos0 + t.token0, p1 = t.pos0 + t.token0 + (t.head0 + t.rows - 1) / G;  // first and last position
    const int lo = a.window > 0 ? max(0, p0 - a.window + 1) : 0;
    if (p1 >= 0) {
        t.step0 = lo / KEYS;
        t.steps = p1 / KEYS + 1 - t.step0;
    }
    t.parts = min(splits, max(1, t.steps / MIN_SPLIT));
    return t;
}

// A step's keys and values on their way from the cache to LDS: 16-byte pieces
// of a thread, unit i of the wave's 1 KiB units.
template <int TYPE, int D, int NW>
struct Stage {
    static constexpr bool FP8 = TYPE == SAE_KV_FP8;
    static constexpr int PAGE = SAE_KV_BLOCK * D * (FP8 ? 1 : 2);  // bytes in the cache
    static constexpr int UNITS = PAGES * PAGE / 1024 / NW;         // units of a wave, of keys and of values each
    static constexpr int PER_PAGE = PAGE / 1024;
    static_assert(UNITS >= 1, "every wave moves something");
    u32x4 k[UNITS], v[UNITS];
    uint32_t ks[UNITS], vs[UNITS][2];
};

// The wave's rows over steps s0 .. s1 - 1 once more, one key at a time on the
// vector units, each row adding the keys it sees and no other: the slow path
// for values that are not finite.  Same state as the loop it replaces.
template <int TYPE, int D>
__device__ void redo(const KvDev &c, const AttnArgs &a, const Tile &t, int64_t base, int kvhead, int s0, int s1, int token,
                     int head, int lo, int pos, f32x16 (&o)[D / 32], float &m, float &l)
{
    constexpr bool FP8 = TYPE == SAE_KV_FP8, F16 = is_f16(TYPE);
    constexpr int E = FP8 ? 1 : 2, PAGE = SAE_KV_BLOCK * D * E, ND = FP8 ? 2 : 1;
    const int h = (int)__lane_id() >> 5;
    const uint16_t *q = static_cast<const uint16_t *>(a.q) + (int64_t)(t.first + token) * a.q_stride + (int64_t)head * D;
    m = NEG_INF;
    l = 0.0f;
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.0f;
#pragma unroll 1
    for (int key = s0 * KEYS; key < min(s1 * KEYS, t.len); ++key) {
        const int id = c.ids[(int64_t)t.seq * c.max_blocks + key / SAE_KV_BLOCK], tk = key % SAE_KV_BLOCK;
        if (base < 0 || id < 0 || id >= c.bpi) continue;  // uniform
        const char *kp = c.k + (base + id) * c.block_bytes + (int64_t)kvhead * PAGE;
        const char *vp = c.v + (base + id) * c.block_bytes + (int64_t)kvhead * PAGE;
        float ks = 1.0f, vs = 1.0f, x = 0.0f;
        if constexpr (FP8) {
            const int64_t sc = (base + id) * c.scale_stride + kvhead * SAE_KV_BLOCK + tk;
            ks = scale_of(c.ks[sc], 0);
            vs = scale_of(c.vs[sc], 0);
        }
#pragma unroll 4
        for (int d = 0; d < D; ++d) {
            float y;
            if constexpr (FP8) y = __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)kp)[d / 16 * 256 + tk * 16 + d % 16], 0);
            else y = low<F16>(((const uint16_t *)kp)[d / 8 * 128 + tk * 8 + d % 8]);
            x = __builtin_fmaf(low<F16>(q[d]), y, x);
        }
        x *= ks * a.scale * LOG2E;
        if (key < lo || key > pos) continue;
        const float mn = fmaxf(m, x), mu = mn == NEG_INF ? 0.0f : mn;
        const float f = exp2_(m - mu), w = exp2_(x - mu);
        m = mn;
        l = l * f + (h == 0 ? w : 0.0f);  // the halves' sums are added at the end
#pragma unroll
        for (int b = 0; b < D / 32; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int d = b * 32 + i / 4 * 8 + h * 4 + i % 4;
                const int at = (((d / (16 * ND) * 16 + d % 16) * 2 + tk / 4 % 2) * ND + d / 16 % ND) * 8 + tk / 8 * 4 + tk % 4;
                float y;
                if constexpr (FP8) y = __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)vp)[at], 0) * vs;
                else y = low<F16>(((const uint16_t *)vp)[at]);
                o[b][i] = __builtin_fmaf(w, y, o[b][i] * f);
                if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // few loads at a time: registers
            }
    }
}

template <int TYPE, int D, int NW>
__global__ void __launch_bounds__(NW * SAE_WAVE, D == 256 ? 1 : 2)
k_prefill(KvDev c, AttnArgs a, Plan plan)
{
    constexpr bool FP8 = TYPE == SAE_KV_FP8, F16 = is_f16(TYPE);
    constexpr int PB = SAE_KV_BLOCK * D * 2;  // bytes of a page in LDS
    constexpr int NM = D / 16, NB = D / 32;
    typedef Stage<TYPE, D, NW> St;
    __shared__ __align__(16) char lds_k[2][PAGES * PB];
    __shared__ __align__(16) char lds_v[2][PAGES * PB];

    // blocks go round-robin over the XCDs: the key-value head varies fastest, so
    // that the tiles that read the same keys tend to share an L2; long tiles
    // (late ones of a prompt) come first
    const int per = c.kvh * plan.splits;
    const int64_t tile = plan.tiles - 1 - (int64_t)(blockIdx.x / per);
    const int part = blockIdx.x % per / c.kvh, kvhead = blockIdx.x % c.kvh;
    const Tile t = tile_of(c, a, tile, NW * ROWS, plan.splits);
    if (t.none || part >= t.parts) return;
    const int G = a.heads / c.kvh;
    const int lane = (int)__lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / SAE_WAVE);
    const int n = lane & 31, h = lane >> 5;
    const int64_t base = kv::seq_base(c, t.seq);
    const int s0 = t.step0 + (int)((int64_t)t.steps * part / t.parts);
    const int s1 = t.step0 + (int)((int64_t)t.steps * (part + 1) / t.parts);

    // this lane's row
    const int wrow = wave * ROWS, row = wrow + n;
    const bool live = row < t.rows;
    const int token = live ? t.token0 + (t.head0 + row) / G : 0;
    const int head = kvhead * G + (live ? (t.head0 + row) % G : 0);
    const int pos = live ? t.pos0 + token : -1;                   // keys lo .. pos are seen
    const int lo = a.window > 0 ? max(0, pos - a.window + 1) : 0;
    // the wave's first and last position (rows are in order of position)
    const bool full_rows = wrow + ROWS <= t.rows;
    const int wp0 = wrow < t.rows ? t.pos0 + t.token0 + (t.head0 + wrow) / G : -1;
    const int wp1 = wrow < t.rows ? t.pos0 + t.token0 + (t.head0 + min(wrow + ROWS, t.rows) - 1) / G : -1;
    const int wlo1 = a.window > 0 ? max(0, wp1 - a.window + 1) : 0;  // the last row's first key
    const int wlo0 = a.window > 0 ? max(0, wp0 - a.window + 1) : 0;

    const float sl = a.scale == 0.0f ? 1.0f : fabsf(a.scale) * LOG2E;
    u32x4 q[NM];
    {
        // a negative scale is the query's sign, a scale of zero a query of zeros
        const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u, keep = a.scale == 0.0f ? 0u : ~0u;
        const char *qr = static_cast<const char *>(a.q) +
                         ((int64_t)(t.first + token) * a.q_stride + (int64_t)head * D + h * 8) * 2;
#pragma unroll
        for (int i = 0; i < NM; ++i) {
            q[i] = u32x4{0, 0, 0, 0};
            if (live) q[i] = (*reinterpret_cast<const u32x4 *>(qr + i * 32) ^ flip) & keep;
        }
    }
    f32x16 o[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.0f;
    float m = NEG_INF, l = 0.0f;

    // table entries of 16 steps: lane 4 j + p has page p of step ids_from + j, -1 for none
    int ids = -1, ids_from = 0;
    auto fetch_ids = [&](int step) {
        ids_from = step;
        const int page = step * PAGES + lane;
        ids = -1;
        if (page * SAE_KV_BLOCK < t.len && step + lane / PAGES < s1) ids = c.ids[(int64_t)t.seq * c.max_blocks + page];
        if (ids >= c.bpi) kv::report(c);
        if (base < 0 || ids >= c.bpi) ids = -1;
    };
    St st;
    auto load = [&](int step) {
        if (step >= s1) return;
        if (step >= ids_from + SAE_WAVE / PAGES) fetch_ids(step);
#pragma unroll
        for (int i = 0; i < St::UNITS; ++i) {
            const int unit = wave * St::UNITS + i, p = unit / St::PER_PAGE;
            const int id = __builtin_amdgcn_readlane(ids, (step - ids_from) * PAGES + p);
            const int64_t blk = id < 0 ? 0 : base + id;
            const int64_t at = blk * c.block_bytes + (int64_t)kvhead * St::PAGE + unit % St::PER_PAGE * 1024 + lane * 16;
            st.k[i] = *reinterpret_cast<const u32x4 *>(c.k + at);
            st.v[i] = *reinterpret_cast<const u32x4 *>(c.v + at);
            if constexpr (FP8) {
                const int64_t sc = blk * c.scale_stride + kvhead * SAE_KV_BLOCK;
                st.ks[i] = c.ks[sc + (lane & 15)];
                st.vs[i][0] = *reinterpret_cast<const uint32_t *>(c.vs + sc + (lane & 1) * 4);
                st.vs[i][1] = *reinterpret_cast<const uint32_t *>(c.vs + sc + (lane & 1) * 4 + 8);
            }
        }
    };
    // Stage -> LDS buffer; what is past the sequence's end or has no block becomes
    // zeros in the values (it may be NaN); such keys' scores are masked later.
    auto store = [&](int step, int buf) {
        if (step >= s1) return;
#pragma unroll
        for (int i = 0; i < St::UNITS; ++i) {
            const int unit = wave * St::UNITS + i, p = unit / St::PER_PAGE, sub = unit % St::PER_PAGE;
            const int id = __builtin_amdgcn_readlane(ids, (step - ids_from) * PAGES + p);
            const int t0 = step * KEYS + p * SAE_KV_BLOCK;
            // bit j: token j of a value piece's 8 is there
            uint32_t keep = 0xFF;
            if (id < 0 || t0 + SAE_KV_BLOCK > t.len) {  // uniform
                keep = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (id >= 0 && t0 + (lane & 1) * 4 + (j >> 2) * 8 + (j & 3) < t.len) keep |= 1u << j;
            }
            if constexpr (FP8) {
                // keys: 16 dimensions of token lane % 16; values: 8 tokens of two dimensions
                char *to = lds_k[buf] + p * PB + (sub * 4 + (lane >> 4)) * 512 + (lane & 15) * 16;
                const float ks = scale_of(st.ks[i], 0);
                *reinterpret_cast<u32x4 *>(to) = widen8(st.k[i][0], st.k[i][1], ks);
                *reinterpret_cast<u32x4 *>(to + 256) = widen8(st.k[i][2], st.k[i][3], ks);
                char *tv = lds_v[buf] + p * PB + (sub * 2 + (lane >> 5)) * 1024 + (lane >> 1 & 15) * 32 + (lane & 1) * 16;
#pragma unroll
                for (int dd = 0; dd < 2; ++dd) {
                    u32x4 w;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {  // tokens 2 j, 2 j + 1 of the piece
                        const uint32_t x = st.v[i][dd * 2 + j / 2] >> (16 * (j & 1));
                        float f0 = __builtin_amdgcn_cvt_f32_fp8((int)x, 0) * scale_of(st.vs[i][j / 2], 2 * (j & 1));
                        float f1 = __builtin_amdgcn_cvt_f32_fp8((int)x, 1) * scale_of(st.vs[i][j / 2], 2 * (j & 1) + 1);
                        if (!(keep >> (2 * j) & 1)) f0 = 0.0f;
                        if (!(keep >> (2 * j + 1) & 1)) f1 = 0.0f;
                        w[j] = pack2<false>(f0, f1);
                    }
                    *reinterpret_cast<u32x4 *>(tv + dd * 512) = w;
                }
            } else {
                const int to = p * PB + sub * 1024 + lane * 16;
                u32x4 w = st.v[i];
                if (keep != 0xFF) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        w[j] &= (keep >> (2 * j) & 1 ? 0xFFFFu : 0u) | (keep >> (2 * j + 1) & 1 ? 0xFFFF0000u : 0u);
                }
                *reinterpret_cast<u32x4 *>(lds_k[buf] + to) = st.k[i];
                *reinterpret_cast<u32x4 *>(lds_v[buf] + to) = w;
            }
        }
    };

    auto compute = [&](int step, int buf, uint32_t holes) {
        const int t0 = step * KEYS;
        if (t0 > wp1 || t0 + KEYS <= wlo0) return;  // no row of the wave sees a key of the step
        f32x16 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[u][i] = 0.0f;
            const char *kp = lds_k[buf] + (u * 2 + (n >> 4)) * PB + h * 256 + (n & 15) * 16;
#pragma unroll
            for (int i = 0; i < NM; ++i) s[u] = mfma32<F16>(*reinterpret_cast<const u32x4 *>(kp + i * 512), q[i], s[u]);
        }
        const bool masked = holes != 0 || !full_rows || t0 + KEYS - 1 > wp0 || t0 < wlo1;  // uniform
        if (masked) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int p = u * 2 + i / 8;
                    const int key = t0 + p * SAE_KV_BLOCK + (i / 4 % 2) * 8 + h * 4 + i % 4;
                    if (key < lo || key > pos) s[u][i] = NEG_INF;
                }
            if (holes) {
#pragma unroll
                for (int p = 0; p < PAGES; ++p)
                    if (holes >> p & 1) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) s[p / 2][p % 2 * 8 + i] = NEG_INF;
                    }
            }
        }
        float top = s[0][0];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[u][i]);
        top = max_halves(top) * sl;
        if (__any(top > m + SLACK)) {
            const float mn = fmaxf(m, top);
            const float f = mn == NEG_INF ? 0.0f : exp2_(m - mn);
            m = mn;
            l *= f;
#pragma unroll
            for (int b = 0; b < NB; ++b) o[b] *= f;
        }
        const float mu = m == NEG_INF ? 0.0f : -m;
        u32x4 w[PAGES];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float x = exp2_(__builtin_fmaf(s[u][i], sl, mu)), y = exp2_(__builtin_fmaf(s[u][i + 1], sl, mu));
                l += x;
                l += y;
                w[u * 2 + i / 8][i / 2 % 4] = pack2<F16>(x, y);
            }
        const char *vp = lds_v[buf] + n * 32 + h * 16;
#pragma unroll
        for (int p = 0; p < PAGES; ++p)
#pragma unroll
            for (int b = 0; b < NB; ++b)
                o[b] = mfma32<F16>(*reinterpret_cast<const u32x4 *>(vp + p * PB + b * 1024), w[p], o[b]);
    };
    // bit p: page p of the step has no block
    auto holes_of = [&](int step) {
        return (uint32_t)(__ballot(ids < 0) >> ((step - ids_from) * PAGES)) & ((1u << PAGES) - 1);
    };

    if (s0 < s1) {
        fetch_ids(s0);
        load(s0);
        store(s0, 0);
        uint32_t holes = holes_of(s0);
        for (int step = s0; step < s1; ++step) {
            const int buf = (step - s0) & 1;
            barrier();       // buffer buf is whole; the other one has been read
            load(step + 1);  // may replace the table entries
            compute(step, buf, holes);
            if (step + 1 < s1) {
                holes = holes_of(step + 1);
                store(step + 1, buf ^ 1);
            }
        }
    }

    // A value that is infinite or NaN reaches, as 0 times itself, also rows that do
    // not see its key.  Only outputs can show that (weights are a row's own).
    bool odd = false;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd |= !(fabsf(o[b][i]) < __builtin_inff());
    if (__any(odd && l < __builtin_inff())) redo<TYPE, D>(c, a, t, base, kvhead, s0, s1, token, head, lo, pos, o, m, l);

    l += __shfl_xor(l, 32);
    if (t.parts == 1) {
        if (!live) return;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;  // no key seen, or every score -inf
        char *to = static_cast<char *>(a.out) + ((int64_t)(t.first + token) * a.out_stride + (int64_t)head * D + h * 4) * 2;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<u32x2 *>(to + (b * 32 + i * 2) * 2) =
                    u32x2{pack2<F16>(o[b][i] * inv, o[b][i + 1] * inv), pack2<F16>(o[b][i + 2] * inv, o[b][i + 3] * inv)};
        if (a.lse && h == 0)
            a.lse[(int64_t)(t.first + token) * a.heads + head] = l == 0.0f ? NEG_INF : (m + log2_(l)) * LN2;
        return;
    }
    // a part: maxima, sums and outputs as the lanes hold them
    const int64_t slot = ((tile * c.kvh + kvhead) * plan.splits + part) * NW + wave;
    float *to = static_cast<float *>(a.work) + slot * (ROWS * (D + 4)) + lane * 4;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<f32x4 *>(to + (b * 4 + i) * 256) = f32x4{o[b][i * 4], o[b][i * 4 + 1], o[b][i * 4 + 2], o[b][i * 4 + 3]};
    float *ml = static_cast<float *>(a.work) + slot * (ROWS * (D + 4)) + ROWS * D + lane * 2;
    *reinterpret_cast<float2 *>(ml) = float2{m, l};
}

// Adds a tile's parts, in order: lanes hold what they held in k_prefill, a wave
// one 32-dimension block of 32 rows.
template <int TYPE, int D, int NW>
__global__ void __launch_bounds__(SAE_WAVE) k_prefill_join(KvDev c, AttnArgs a, Plan plan)
{
    constexpr bool F16 = is_f16(TYPE);
    const int wave = blockIdx.y % NW, b = blockIdx.y / NW;
    const int64_t tile = blockIdx.x / c.kvh;
    const int kvhead = blockIdx.x % c.kvh, G = a.heads / c.kvh;
    const Tile t = tile_of(c, a, tile, NW * ROWS, plan.splits);
    if (t.none || t.parts == 1) return;
    const int lane = (int)__lane_id(), n = lane & 31, h = lane >> 5;
    const int row = wave * ROWS + n;
    const bool live = row < t.rows;
    if (!__any(live)) return;
    const float *from = static_cast<const float *>(a.work) + ((tile * c.kvh + kvhead) * plan.splits * NW + wave) * (ROWS * (D + 4));
    const int64_t stride = (int64_t)NW * (ROWS * (D + 4));
    float m = NEG_INF, l = 0.0f;
    f32x4 o[4] = {};
    for (int p = 0; p < t.parts; ++p, from += stride) {
        const float2 ml = *reinterpret_cast<const float2 *>(from + ROWS * D + lane * 2);
        f32x4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const f32x4 *>(from + (b * 4 + i) * 256 + lane * 4);
        const float top = fmaxf(m, ml.x), mu = top == NEG_INF ? 0.0f : top;
        const float f0 = exp2_(m - mu), f1 = exp2_(ml.x - mu);
        l = l * f0 + ml.y * f1;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = o[i] * f0 + x[i] * f1;
        m = top;
    }
    if (!live) return;
    const int token = t.token0 + (t.head0 + row) / G, head = kvhead * G + (t.head0 + row) % G;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    char *to = static_cast<char *>(a.out) + ((int64_t)(t.first + token) * a.out_stride + (int64_t)head * D + b * 32 + h * 4) * 2;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        *reinterpret_cast<u32x2 *>(to + i * 16) =
            u32x2{pack2<F16>(o[i][0] * inv, o[i][1] * inv), pack2<F16>(o[i][2] * inv, o[i][3] * inv)};
    if (a.lse && h == 0 && b == 0)
        a.lse[(int64_t)(t.first + token) * a.heads + head] = l == 0.0f ? NEG_INF : (m + log2_(l)) * LN2;
}

constexpr int WAVES = 4;

Plan plan_of(const KvDev &c, int n_tokens, int heads, int kvh)
{
    Plan p;
    const int G = heads / kvh;
    p.tiles = c.qs ? (int)((int64_t)n_tokens * G / (WAVES * ROWS)) + c.n_seq : c.n_seq * ((G + WAVES * ROWS - 1) / (WAVES * ROWS));
    const int64_t items = (int64_t)p.tiles * kvh;
    p.splits = items >= GROUPS ? 1 : (int)(GROUPS / items);
    return p;
}

template <int TYPE, int D>
hipError_t launch(const KvDev &c, const AttnArgs &a, hipStream_t s)
{
    const Plan p = plan_of(c, c.n_tokens, a.heads, c.kvh);
    hipLaunchKernelGGL((k_prefill<TYPE, D, WAVES>), dim3(p.tiles * c.kvh * p.splits), dim3(WAVES * SAE_WAVE), 0, s, c, a, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    hipLaunchKernelGGL((k_prefill_join<TYPE, D, WAVES>), dim3(p.tiles * c.kvh, WAVES * (D / 32)), dim3(SAE_WAVE), 0, s, c, a, p);
    return hipGetLastError();
}

template <int TYPE>
hipError_t launch_dim(const KvDev &c, const AttnArgs &a, int dim, hipStream_t s)
{
    return dim == 64 ? launch<TYPE, 64>(c, a, s) : dim == 128 ? launch<TYPE, 128>(c, a, s) : launch<TYPE, 256>(c, a, s);
}

}  // namespace

// Enough for every call: there are parts only where all workgroups are at most GROUPS.
size_t prefill_work_bytes(int dim) { return (size_t)GROUPS * WAVES * ROWS * (dim + 4) * sizeof(float); }

// Whether the call's tiles fit one launch.
bool prefill_fits(const KvDev &c, int heads)
{
    const int64_t G = heads / c.kvh, rows = WAVES * ROWS;
    const int64_t tiles = c.qs ? c.n_tokens * G / rows + c.n_seq : c.n_seq * ((G + rows - 1) / rows);
    return tiles * c.kvh < (1ll << 23);
}

hipError_t launch_prefill(const KvDev &c, const AttnArgs &a, int type, int dim, hipStream_t s)
{
    if (type == SAE_KV_BF16) return launch_dim<SAE_KV_BF16>(c, a, dim, s);
    if (type == SAE_KV_F16) return launch_dim<SAE_KV_F16>(c, a, dim, s);
    return launch_dim<SAE_KV_FP8>(c, a, dim, s);
}
