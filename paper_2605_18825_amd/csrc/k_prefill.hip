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
#include <algorithm>

#include "attn_tile.h"

namespace {

using namespace attn;

constexpr int ROWS = 32;   // rows of a wave
// Keys of a step: 64, or 32 where a row's state and a step's scores would not fit
// the registers together.
constexpr int keys_of(int dim) { return dim == 256 ? 32 : 64; }
constexpr int MIN_SPLIT = 128;   // keys of a split at least
// Workgroups wanted: two per compute unit, one of the larger heads.
constexpr int groups_of(int dim) { return dim == 256 ? 256 : 512; }
constexpr float SLACK = 8.0f;    // of the running maximum, in powers of two

// Everything written to LDS before it, by stores or by to_lds(), is whole after it.
__device__ __forceinline__ void barrier()
{
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): to_lds() has arrived
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// 16 bytes per lane from memory to LDS, lane l's to `to` + 16 l.
__device__ __forceinline__ void to_lds(const char *from, char *to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                     (__attribute__((address_space(3))) void *)to, 16, 0, 0);
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
    int step0, steps;      // steps of keys_of(dim) keys the tile sees: step0 .. step0 + steps - 1
    int parts;             // workgroups they are divided over
    bool none;
};

__device__ __forceinline__ Tile tile_of(const KvDev &c, const AttnArgs &a, int64_t tile, int rows, int splits, int keys)
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
        t.step0 = lo / keys;
        t.steps = p1 / keys + 1 - t.step0;
    }
    t.parts = min(splits, max(1, t.steps / (MIN_SPLIT / keys)));
    return t;
}

// A step's keys or values on their way from the cache to LDS: 16-byte pieces of
// a thread, unit i of the wave's 1 KiB units.
template <int TYPE, int D, int NW>
struct Stage {
    static constexpr bool FP8 = TYPE == SAE_KV_FP8;
    static constexpr int PAGE = SAE_KV_BLOCK * D * (FP8 ? 1 : 2);  // bytes in the cache
    static constexpr int UNITS = keys_of(D) / SAE_KV_BLOCK * PAGE / 1024 / NW;         // units of a wave
    static constexpr int PER_PAGE = PAGE / 1024;
    static_assert(UNITS >= 1, "every wave moves something");
    u32x4 x[UNITS];
    uint32_t s[UNITS][2];  // scale bytes of an 8-bit cache
};

// The wave's rows over steps s0 .. s1 - 1 once more, one key at a time on the
// vector units, each row adding the keys it sees and no other: the slow path
// for values that are not finite.  Same state as the loop it replaces.
template <int TYPE, int D>
__device__ void redo(const KvDev &c, const AttnArgs &a, const Tile &t, int64_t base, int kvhead, int s0, int s1, int token,
                     int head, int pos, f32x16 (&o)[D / 32], float &m, float &l)
{
    constexpr bool FP8 = TYPE == SAE_KV_FP8, F16 = is_f16(TYPE);
    constexpr int E = FP8 ? 1 : 2, PAGE = SAE_KV_BLOCK * D * E, ND = FP8 ? 2 : 1, KEYS = keys_of(D);
    const int h = (int)__lane_id() >> 5, lo = a.window > 0 ? max(0, pos - a.window + 1) : 0;
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

// The end of a tile's part: outputs where it is the only one.
template <int TYPE, int D, int NW>
__device__ __forceinline__ void finish(const KvDev &c, const AttnArgs &a, const Plan &plan, const Tile &t, int64_t base,
                                       int kvhead, int wave, int64_t tile, int part, int s0, int s1, f32x16 (&o)[D / 32],
                                       float m, float l)
{
    constexpr bool F16 = is_f16(TYPE);
    constexpr int NB = D / 32;
    const int G = a.heads / c.kvh;
    // the lane's number as if it were not known before: what is derived from it need
    // not be kept in registers through the steps
    int lane = (int)__lane_id();
    asm volatile("" : "+v"(lane));
    const int h = lane >> 5, row = wave * ROWS + (lane & 31);
    const bool live = row < t.rows;
    const int token = live ? t.token0 + (t.head0 + row) / G : 0, head = kvhead * G + (live ? (t.head0 + row) % G : 0);
    // A value that is infinite or NaN reaches, as 0 times itself, also rows that do
    // not see its key.  Only outputs can show that (weights are a row's own).
    bool odd = false;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd |= !(fabsf(o[b][i]) < __builtin_inff());
    if (__any(odd && l < __builtin_inff())) redo<TYPE, D>(c, a, t, base, kvhead, s0, s1, token, head, live ? t.pos0 + token : -1, o, m, l);

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

template <int TYPE, int D, int NW>
__global__ void __launch_bounds__(NW * SAE_WAVE, D == 256 ? 1 : 2)
k_prefill(KvDev c, AttnArgs a, Plan plan)
{
    constexpr bool FP8 = TYPE == SAE_KV_FP8, F16 = is_f16(TYPE);
    constexpr int PB = SAE_KV_BLOCK * D * 2;  // bytes of a page in LDS
    constexpr int KEYS = keys_of(D), PAGES = KEYS / SAE_KV_BLOCK, KT = KEYS / 32;
    constexpr int NM = D / 16, NB = D / 32;
    // LDS reads in flight while as many products are taken (an 8-bit cache's stage
    // leaves fewer registers)
    constexpr int BATCH = FP8 ? 2 : 4;
    typedef Stage<TYPE, D, NW> St;
    // arrays of their own: the compiler then sees that a read of one does not depend
    // on loads into another
    __shared__ __align__(16) char k_even[PAGES * PB], k_odd[PAGES * PB], v_even[PAGES * PB], v_odd[PAGES * PB];
    char *const lds_k[2] = {k_even, k_odd}, *const lds_v[2] = {v_even, v_odd};

    // blocks go round-robin over the XCDs: the key-value head varies fastest, so
    // that the tiles that read the same keys tend to share an L2; long tiles
    // (late ones of a prompt) come first
    const int per = c.kvh * plan.splits;
    const int64_t tile = plan.tiles - 1 - (int64_t)(blockIdx.x / per);
    const int part = blockIdx.x % per / c.kvh, kvhead = blockIdx.x % c.kvh;
    const Tile t = tile_of(c, a, tile, NW * ROWS, plan.splits, keys_of(D));
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
    const int pos = live ? t.pos0 + t.token0 + (t.head0 + row) / G : -1;  // keys lo .. pos are seen
    const int lo = a.window > 0 ? max(0, pos - a.window + 1) : 0;
    // the wave's first and last position (rows are in order of position)
    const bool full_rows = wrow + ROWS <= t.rows;
    const int wp0 = wrow < t.rows ? t.pos0 + t.token0 + (t.head0 + wrow) / G : -1;
    const int wp1 = wrow < t.rows ? t.pos0 + t.token0 + (t.head0 + min(wrow + ROWS, t.rows) - 1) / G : -1;
    const int wlo1 = a.window > 0 ? max(0, wp1 - a.window + 1) : 0;  // the last row's first key

    const float sl = a.scale == 0.0f ? 1.0f : fabsf(a.scale) * LOG2E;
    u32x4 q[NM];
    {
        // a negative scale is the query's sign, a scale of zero a query of zeros
        const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u, keep = a.scale == 0.0f ? 0u : ~0u;
        const int token = live ? t.token0 + (t.head0 + row) / G : 0, head = kvhead * G + (live ? (t.head0 + row) % G : 0);
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
    // bit p: page p of the step has no block
    auto holes_of = [&](int step) {
        return (uint32_t)(__ballot(ids < 0) >> ((step - ids_from) * PAGES)) & ((1u << PAGES) - 1);
    };
    // the cache block and place of the wave's unit i of a step
    auto unit_block = [&](int step, int i, int &sub) {
        const int unit = wave * St::UNITS + i;
        sub = unit % St::PER_PAGE;
        const int id = __builtin_amdgcn_readlane(ids, (step - ids_from) * PAGES + unit / St::PER_PAGE);
        return id < 0 ? 0 : base + id;
    };
    // Value pieces (16 bytes: half h of dimension n of 32) lie in LDS at piece 2 n + h
    // with its lowest bit flipped by bit 4: the lanes that LDS serves together then
    // read all banks (without the flip two of them met in each).
    const int flip = lane ^ (lane >> 4 & 1);
    // A step's keys or values into LDS: 16-bit ones go there directly, 8-bit ones
    // through registers.  What is there is whole after the next barrier().
    auto load_k1 = [&](int step, St &st, char *to, int i) __attribute__((always_inline)) {
        int sub;
        const int64_t blk = unit_block(step, i, sub);
        const char *from = c.k + (blk * c.block_bytes + (int64_t)kvhead * St::PAGE + sub * 1024) + (uint32_t)lane * 16u;
        if constexpr (FP8) {
            st.x[i] = *reinterpret_cast<const u32x4 *>(from);
            st.s[i][0] = c.ks[blk * c.scale_stride + kvhead * SAE_KV_BLOCK + (lane & 15)];
        } else {
            to_lds(from, to + (wave * St::UNITS + i) * 1024);
        }
    };
    auto load_v1 = [&](int step, St &st, char *to, int i) __attribute__((always_inline)) {
        int sub;
        const int64_t blk = unit_block(step, i, sub);
        const char *from = c.v + (blk * c.block_bytes + (int64_t)kvhead * St::PAGE + sub * 1024);
        if constexpr (FP8) {
            st.x[i] = *reinterpret_cast<const u32x4 *>(from + (uint32_t)lane * 16u);
            const uint8_t *sc = c.vs + blk * c.scale_stride + kvhead * SAE_KV_BLOCK + (lane & 1) * 4;
            st.s[i][0] = *reinterpret_cast<const uint32_t *>(sc);
            st.s[i][1] = *reinterpret_cast<const uint32_t *>(sc + 8);
        } else {
            to_lds(from + (uint32_t)flip * 16u, to + (wave * St::UNITS + i) * 1024);
        }
    };
    auto load_k = [&](int step, St &st, char *to) {
#pragma unroll
        for (int i = 0; i < St::UNITS; ++i) load_k1(step, st, to, i);
    };
    auto load_v = [&](int step, St &st, char *to) {
#pragma unroll
        for (int i = 0; i < St::UNITS; ++i) load_v1(step, st, to, i);
    };
    auto store_k = [&](const St &st, char *lds) {
        if constexpr (FP8) {
#pragma unroll
            for (int i = 0; i < St::UNITS; ++i) {  // 16 dimensions of token lane % 16
                const int unit = wave * St::UNITS + i, p = unit / St::PER_PAGE, sub = unit % St::PER_PAGE;
                char *to = lds + p * PB + (sub * 4 + (lane >> 4)) * 512 + (lane & 15) * 16;
                const float ks = scale_of(st.s[i][0], 0);
                *reinterpret_cast<u32x4 *>(to) = widen8(st.x[i][0], st.x[i][1], ks);
                *reinterpret_cast<u32x4 *>(to + 256) = widen8(st.x[i][2], st.x[i][3], ks);
            }
        }
    };
    auto store_v = [&](const St &st, char *lds) {
        if constexpr (FP8) {
#pragma unroll
            for (int i = 0; i < St::UNITS; ++i) {  // 8 tokens of two dimensions
                const int unit = wave * St::UNITS + i, p = unit / St::PER_PAGE, sub = unit % St::PER_PAGE;
#pragma unroll
                for (int dd = 0; dd < 2; ++dd) {
                    u32x4 w;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {  // tokens 2 j, 2 j + 1 of the piece
                        const uint32_t x = st.x[i][dd * 2 + j / 2] >> (16 * (j & 1));
                        w[j] = pack2<false>(__builtin_amdgcn_cvt_f32_fp8((int)x, 0) * scale_of(st.s[i][j / 2], 2 * (j & 1)),
                                            __builtin_amdgcn_cvt_f32_fp8((int)x, 1) * scale_of(st.s[i][j / 2], 2 * (j & 1) + 1));
                    }
                    *reinterpret_cast<u32x4 *>(lds + p * PB + (sub * 2 + (lane >> 5)) * 1024 + dd * 512 + (flip & 31) * 16) = w;
                }
            }
        }
    };
    // Zeros in the values of keys past the sequence's end or without a block (they
    // may be NaN; their scores are masked).  The whole workgroup, or none of it.
    auto clean_v = [&](int step, uint32_t holes, char *lds) {
        if (holes == 0 && (step + 1) * KEYS <= t.len) return;
        for (int i = threadIdx.x; i < PAGES * PB / 16; i += NW * SAE_WAVE) {
            const int p = i / (PB / 16), piece = i % 64 ^ (i >> 4 & 1);
            u32x4 w = *reinterpret_cast<u32x4 *>(lds + i * 16);
#pragma unroll
            for (int j = 0; j < 8; ++j) {  // token j of the piece's 8
                const int key = step * KEYS + p * SAE_KV_BLOCK + (piece & 1) * 4 + (j >> 2) * 8 + (j & 3);
                if (key >= t.len || (holes >> p & 1)) w[j / 2] &= j & 1 ? 0xFFFFu : 0xFFFF0000u;
            }
            *reinterpret_cast<u32x4 *>(lds + i * 16) = w;
        }
        barrier();
    };

    const int kfrag = (n >> 4) * PB + h * 256 + (n & 15) * 16, vfrag = ((n * 2 + h) ^ (n >> 3 & 1)) * 16;
    auto scores = [&](f32x16 (&s)[KT], int buf) {
        const char *kp = lds_k[buf] + kfrag;
#pragma unroll
        for (int u = 0; u < KT; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[u][i] = 0.0f;
#pragma unroll
        for (int i = 0; i < NM; ++i)
#pragma unroll
            for (int u = 0; u < KT; ++u)
                s[u] = mfma32<F16>(*reinterpret_cast<const u32x4 *>(kp + u * 2 * PB + i * 512), q[i], s[u]);
    };
    auto mask = [&](f32x16 (&s)[KT], int step, uint32_t holes) {
        const int t0 = step * KEYS;
        if (holes == 0 && full_rows && t0 + KEYS - 1 <= wp0 && t0 >= wlo1) return;  // uniform
        asm volatile("");  // a branch: the comparisons are not worth taking on every step
#pragma unroll
        for (int u = 0; u < KT; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int p = u * 2 + i / 8;
                const int key = t0 + p * SAE_KV_BLOCK + (i / 4 % 2) * 8 + h * 4 + i % 4;
                if (key < lo || key > pos || (holes >> p & 1)) s[u][i] = NEG_INF;
            }
    };
    // The maximum of a step's scores, in powers of two.
    auto maximum = [&](const f32x16 (&s)[KT]) {
        float top = s[0][0];
#pragma unroll
        for (int u = 0; u < KT; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[u][i]);
        return max_halves(top) * sl;
    };
    // Follows the maximum: outputs and sums shrink where it grew by more than SLACK.
    auto follow = [&](float top) {
        if (!__any(top > m + SLACK)) return;
        const float mn = fmaxf(m, top);
        const float f = mn == NEG_INF ? 0.0f : exp2_(m - mn);
        m = mn;
        l *= f;
#pragma unroll
        for (int b = 0; b < NB; ++b) o[b] *= f;
    };
    auto weights = [&](const f32x16 (&s)[KT], u32x4 (&w)[PAGES]) {
        const float mu = m == NEG_INF ? 0.0f : -m;
#pragma unroll
        for (int u = 0; u < KT; ++u)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float x = exp2_(__builtin_fmaf(s[u][i], sl, mu)), y = exp2_(__builtin_fmaf(s[u][i + 1], sl, mu));
                l += x;
                l += y;
                w[u * 2 + i / 8][i / 2 % 4] = pack2<F16>(x, y);
            }
    };
    auto outputs = [&](const u32x4 (&w)[PAGES], int buf) {
        const char *vp = lds_v[buf] + vfrag;
#pragma unroll
        for (int p = 0; p < PAGES; ++p)
#pragma unroll
            for (int b = 0; b < NB; ++b)
                o[b] = mfma32<F16>(*reinterpret_cast<const u32x4 *>(vp + p * PB + b * 1024), w[p], o[b]);
    };

    if (s0 < s1) {
        // Step t's weights are computed while the matrix units take step t + 1's
        // scores, and that step's maximum while they add step t to the outputs: keys
        // are staged one step ahead of values.
        St sk, sv;
        f32x16 s[KT];
        u32x4 w[PAGES];
        fetch_ids(s0);
        uint32_t holes0 = holes_of(s0), holes = 0;  // of the step whose values, and of the one whose scores come next
        {
            St k0;
            const int next = min(s0 + 1, s1 - 1);
            load_k(s0, k0, k_even);
            load_v(s0, sv, v_even);
            load_k(next, sk, k_odd);
            holes = holes_of(next);
            store_k(k0, k_even);
            store_v(sv, v_even);
            store_k(sk, k_odd);
        }
        barrier();
        scores(s, 0);
        mask(s, s0, holes0);
        follow(maximum(s));
        int step = s0;
        auto body = [&](f32x16 (&s)[KT], f32x16 (&s2)[KT], int buf) __attribute__((always_inline)) {
            // here: s are this step's scores; its values and the next one's keys are in LDS
            clean_v(step, holes0, lds_v[buf]);
            // keys two steps ahead; past the end the last ones again, never used
            const int ahead = min(step + 2, s1 - 1);
            if (ahead >= ids_from + SAE_WAVE / PAGES) fetch_ids(step + 1);
            const uint32_t holes2 = holes_of(ahead);
            if constexpr (FP8) {
                load_k(ahead, sk, nullptr);
                load_v(step + 1, sv, nullptr);
            }
            // Scores 2 j, 2 j + 1 become weights.  A vector operation costs a product less
            // than its own time where every product has a few beside it, and more the more
            // it has: EARLY pairs go with the first products, the others and the maximum
            // with the second.
            constexpr int PAIRS = 8 * KT, EARLY = PAIRS * 3 / 4;
            const float mu = m == NEG_INF ? 0.0f : -m;
            auto pair = [&](int j) __attribute__((always_inline)) {
                const float x = exp2_(__builtin_fmaf(s[j / 8][j % 8 * 2], sl, mu));
                const float y = exp2_(__builtin_fmaf(s[j / 8][j % 8 * 2 + 1], sl, mu));
                l += x;
                l += y;
                uint32_t z = pack2<F16>(x, y);
                asm volatile("" : "+v"(z), "+v"(l));  // here, not where it is used
                w[j / 4][j % 4] = z;
            };
            {
                // products, LDS reads and vector operations in this order
                const char *kp = lds_k[buf ^ 1] + kfrag;
                auto piece = [&](int i) { return *reinterpret_cast<const u32x4 *>(kp + i % KT * 2 * PB + i / KT * 512); };
                u32x4 f[2 * BATCH];
#pragma unroll
                for (int i = 0; i < BATCH; ++i) f[i] = piece(i);
#pragma unroll
                for (int u = 0; u < KT; ++u)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s2[u][i] = 0.0f;
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < NM * KT; ++i) {
                    if (i % BATCH == 0) {
#pragma unroll
                        for (int j = i + BATCH; j < i + 2 * BATCH && j < NM * KT; ++j) f[j % (2 * BATCH)] = piece(j);
                    }
                    s2[i % KT] = mfma32<F16>(f[i % (2 * BATCH)], q[i / KT], s2[i % KT]);
                    if (!FP8 && i * 2 * St::UNITS % (NM * KT) == 0) {  // spread: loads issued at once stall the wave
                        const int u = i * 2 * St::UNITS / (NM * KT);
                        if (u < St::UNITS) load_k1(ahead, sk, lds_k[buf], u);
                        else load_v1(step + 1, sv, lds_v[buf ^ 1], u - St::UNITS);
                    }
#pragma unroll
                    for (int j = i * EARLY / (NM * KT); j < (i + 1) * EARLY / (NM * KT); ++j) pair(j);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            mask(s2, step + 1, holes);
            float top = s2[0][0];
            {
                const char *vp = lds_v[buf] + vfrag;
                auto piece = [&](int i) { return *reinterpret_cast<const u32x4 *>(vp + i / NB * PB + i % NB * 1024); };
                u32x4 f[2 * BATCH];
#pragma unroll
                for (int i = 0; i < BATCH; ++i) f[i] = piece(i);
                __builtin_amdgcn_sched_barrier(0);
                constexpr int N = NB * PAGES, LATE = N / 2;  // the last page's weights are first used after 3 N / 4 products
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if (i % BATCH == 0) {
#pragma unroll
                        for (int j = i + BATCH; j < i + 2 * BATCH && j < N; ++j) f[j % (2 * BATCH)] = piece(j);
                    }
                    o[i % NB] = mfma32<F16>(f[i % (2 * BATCH)], w[i / NB], o[i % NB]);
#pragma unroll
                    for (int j = EARLY + i * (PAIRS - EARLY) / LATE; j < EARLY + (i + 1) * (PAIRS - EARLY) / LATE; ++j)
                        if (i < LATE) pair(j);
#pragma unroll
                    for (int j = (i - LATE / 2) * 16 * KT / (N - LATE / 2); j < (i + 1 - LATE / 2) * 16 * KT / (N - LATE / 2); ++j)
                        if (i >= LATE / 2) top = fmaxf(top, s2[j / 16][j % 16]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            follow(max_halves(top) * sl);
            store_k(sk, lds_k[buf]);
            store_v(sv, lds_v[buf ^ 1]);
            holes0 = holes;
            holes = holes2;
            barrier();  // keys of step + 2 and values of step + 1 are whole, what they replaced was read before
            ++step;
        };
        f32x16 t[KT];
        while (step + 2 < s1) {
            body(s, t, 0);
            body(t, s, 1);
        }
        if (step + 1 < s1) {
            body(s, t, 0);
            clean_v(step, holes0, v_odd);
            weights(t, w);
            outputs(w, 1);
        } else {
            clean_v(step, holes0, v_even);
            weights(s, w);
            outputs(w, 0);
        }
    }

    finish<TYPE, D, NW>(c, a, plan, t, base, kvhead, wave, tile, part, s0, s1, o, m, l);
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
    const Tile t = tile_of(c, a, tile, NW * ROWS, plan.splits, keys_of(D));
    if (t.none || t.parts == 1) return;
    const int lane = (int)__lane_id(), n = lane & 31, h = lane >> 5;
    const int row = wave * ROWS + n;
    const bool live = row < t.rows;
    if (!__any(live)) return;
    const float *from = static_cast<const float *>(a.work) + ((tile * c.kvh + kvhead) * plan.splits * NW + wave) * (ROWS * (D + 4));
    const int64_t stride = (int64_t)NW * (ROWS * (D + 4));
    constexpr int UN = 4;  // parts in flight
    float m = NEG_INF, l = 0.0f;
    f32x4 o[4] = {};
    for (int p = 0; p < t.parts; p += UN) {
        float2 ml[UN];
        f32x4 y[UN][4];
#pragma unroll
        for (int k = 0; k < UN; ++k) {
            const float *at = from + min(p + k, t.parts - 1) * stride;  // past the end: not added below
            ml[k] = *reinterpret_cast<const float2 *>(at + ROWS * D + lane * 2);
#pragma unroll
            for (int e = 0; e < 4; ++e) y[k][e] = *reinterpret_cast<const f32x4 *>(at + (b * 4 + e) * 256 + lane * 4);
        }
#pragma unroll
        for (int k = 0; k < UN; ++k) {
            if (p + k >= t.parts) break;  // uniform
            const float top = fmaxf(m, ml[k].x), mu = top == NEG_INF ? 0.0f : top;
            const float f0 = exp2_(m - mu), f1 = exp2_(ml[k].x - mu);
            l = l * f0 + ml[k].y * f1;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = o[e] * f0 + y[k][e] * f1;
            m = top;
        }
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

Plan plan_of(const KvDev &c, int n_tokens, int heads, int kvh, int dim, int window)
{
    Plan p;
    const int G = heads / kvh;
    p.tiles = c.qs ? (int)((int64_t)n_tokens * G / (WAVES * ROWS)) + c.n_seq : c.n_seq * ((G + WAVES * ROWS - 1) / (WAVES * ROWS));
    const int64_t items = (int64_t)p.tiles * kvh;
    // no tile has more parts than MIN_SPLIT goes into the keys that it can see
    int64_t keys = (int64_t)c.max_blocks * SAE_KV_BLOCK;
    if (window > 0) keys = std::min(keys, (int64_t)window + WAVES * ROWS + keys_of(dim));
    const int64_t most = std::max(std::min((int64_t)groups_of(dim) / std::max(items, (int64_t)1), (keys + keys_of(dim)) / MIN_SPLIT), (int64_t)1);
    p.splits = (int)most;
    return p;
}

template <int TYPE, int D>
hipError_t launch(const KvDev &c, const AttnArgs &a, hipStream_t s)
{
    const Plan p = plan_of(c, c.n_tokens, a.heads, c.kvh, D, a.window);
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

// Enough for every call: there are parts only where all workgroups are at most groups_of(dim).
size_t prefill_work_bytes(int dim) { return (size_t)groups_of(dim) * WAVES * ROWS * (dim + 4) * sizeof(float); }

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
