// Attention of drafted tokens that form trees over the paged key-value cache.
//
// A tree comes as its tokens' parents.  Which tokens a row sees is a row of bits in LDS, made from the
// parents in log2(tokens) rounds (fill_masks) by the workgroups whose keys reach into the tree, or
// that a window's depths matter to; a step of keys takes from it a word or two a row, shifted to the
// step's first key.  Steps before the tree need none.
//
// Rows (tokens x query heads of a key-value head), tiles of 128 of them, their division over
// workgroups, their ends and joins are those of prefill_tile.h, and so is the loop, but for 16-bit caches
// with heads of 64: a step there is 16 KB, too little to be on its way.  Their loop takes keys and
// values through a ring of four stages of 16 KB in LDS, three of them in flight, with one barrier a stage (37
// sequences of up to 201 nodes behind up to 12,000 tokens, window 4,097, 12 heads: 46.7 us by the other loop, 41.3;
// with heads of 128 both take the same: 60 us for 32 sequences of 16..32 nodes behind 512..2,048, 90 for 64 of 2).
//
// Bound by memory (few rows) or by parts of uneven size, their starts and ends: those 32 sequences, 183 MB, take 52 us, for the
// longest part of 16 steps (mean 10.9); 10 are a workgroup's start (its part found, 2 us; table, queries and first keys, 3; the tree,
// 1) and end, and 5 more the join.  The ragged batch above is 780 workgroups, two rounds, of up to 17 steps, mean 8.5.  Wide
// trees are bound by products: 64 nodes behind 16,385..32,768 tokens of an 8-bit cache, 28 heads on 4, 0.70
// PFLOP/s.  Built and taken out: all rows in each wave's registers and keys straight from memory to them (k_decode.hip's
// way): 10 % faster with 8 rows, as fast with 32, 73 us instead of 54 with 64.
#include "prefill_tile.h"

namespace {

constexpr int STAGES = 4;
constexpr int stage_keys(int dim) { return 8192 / (dim * 2); }  // 8 KB of keys, 8 KB of values

// 16 bytes per lane from memory to LDS, lane l's to `to` + 16 l, with nothing that the compiler would wait for by
// itself: it takes every read of LDS for one of what such a load brings, and would wait for the stages ahead (53.3 us
// for the ragged batch above).  m0 (the address, read as the load issues) is left as it was: the compiler takes it for reserved and
// does not heed it among the clobbers, and may keep an address of its own there for such loads as to_lds().
__device__ __forceinline__ void ring_load(const char *from, char *to)
{
    const uint32_t at = (uint32_t)uniform((int)(uintptr_t)(__attribute__((address_space(3))) char *)to);
    uint32_t held;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(held) : "s"(at), "v"(from) : "memory");
}

// A barrier at which all but the wave's `LATER` newest loads have arrived, and what it read from LDS or wrote there.
template <int LATER>
__device__ __forceinline__ void ring_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(LATER) : "memory");
}

template <int TYPE, int D, bool SPLIT>
__global__ void __launch_bounds__(WAVES * SAE_WAVE, 2) k_tree_ring(KvDev c, AttnArgs a, Plan plan)
{
    constexpr int NW = WAVES;
    constexpr bool F16 = is_f16(TYPE);
    constexpr int PB = SAE_KV_BLOCK * D * 2;  // bytes of a page
    constexpr int KEYS = keys_of(D), SK = stage_keys(D), PER_STEP = KEYS / SK;  // keys of a step, of a stage
    constexpr int PAGES = SK / SAE_KV_BLOCK, KT = SK / 32;
    constexpr int NM = D / 16, NB = D / 32;
    constexpr int UNITS = PAGES * PB / 1024 / NW, PER_PAGE = PB / 1024;  // 1 KB pieces of a wave, of keys and of values
    constexpr int ENTRIES = SAE_WAVE / PAGES;                            // stages whose table entries a wave holds
    static_assert(UNITS == 2 && KT >= 1, "a stage is 16 KB");
    // arrays of their own: a read of one does not depend on loads into another
    constexpr int V = PAGES * PB;  // values lie behind the keys
    __shared__ __align__(16) char r0[2 * V], r1[2 * V], r2[2 * V], r3[2 * V];
    __shared__ Masks masks;

    const int x = blockIdx.x / c.kvh, kvhead = blockIdx.x % c.kvh, G = a.heads / c.kvh;
    Tile t;
    int part = 0, nparts = 1, slot = x;
    if constexpr (SPLIT) {
        const Part p = find_part_tree<NW>(c, a, plan, x, NW * ROWS, KEYS);
        if (p.seq >= 0) t = tile_of<true>(c, a, p.seq, p.sub, NW * ROWS, KEYS);
        note_split(a, plan, p, t, kvhead);
        if (p.seq < 0) return;
        part = p.part;
        nparts = p.parts;
        slot = p.slot;
    } else {
        t = find_tile<true>(c, a, plan.tiles - 1 - x, NW * ROWS, KEYS);
    }
    if (t.rows == 0) return;
    const int lane = (int)__lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / SAE_WAVE);
    const int n = lane & 31, h = lane >> 5;
    const int64_t base = kv::seq_base(c, t.seq);
    const int s0 = t.step0 + (int)((int64_t)t.steps * part / nparts);
    const int s1 = t.step0 + (int)((int64_t)t.steps * (part + 1) / nparts);
    const int first = s0 * PER_STEP;
    const int last = min(s1 * PER_STEP, (t.len + SK - 1) / SK);  // stages first .. last - 1
    int parent = -1;
    if (t.tokens > a.max_nodes && threadIdx.x == 0 && c.status) atomicOr(c.status, (uint32_t)SAE_ST_BAD_TREE);
    if (t.tokens <= a.max_nodes && (int)threadIdx.x < t.tokens) parent = a.parent[t.first + threadIdx.x];

    // table entries: lane PAGES j + p has page p of stage ids_from + j, -1 for none
    int ids = -1, ids_from = 0;
    auto load_ids = [&](int stage) __attribute__((always_inline)) {
        ids_from = stage;
        const int page = stage * PAGES + lane;
        ids = -1;
        if (page * SAE_KV_BLOCK < t.len && stage + lane / PAGES < last) ids = c.ids[(int64_t)t.seq * c.max_blocks + page];
    };
    auto check_ids = [&]() __attribute__((always_inline)) {
        if (ids >= c.bpi) kv::report(c);
        if (base < 0 || ids >= c.bpi) ids = -1;
    };
    load_ids(first);
    __builtin_amdgcn_sched_barrier(0);

    // this lane's row
    const int wrow = wave * ROWS, row = wrow + n;
    const bool live = row < t.rows;
    const int token = live ? t.token0 + (t.head0 + row) / G : 0, head = kvhead * G + (live ? (t.head0 + row) % G : 0);
    const int pos = live ? t.pos0 + token : -1;
    int lo = pos < 0 ? 1 << 30 : 0;          // the first key it sees
    const int tree0 = max(t.pos0, 0);
    // keys from all0 to before all1 are seen by all rows of the tile
    const int all0 = a.window > 0 ? max(0, t.pos0 + t.token0 + (t.head0 + t.rows - 1) / G - a.window + 1) : 0;
    const int all1 = t.pos0 + t.token0 >= 0 ? tree0 : 0;
    const float sl = a.scale == 0.0f ? 1.0f : fabsf(a.scale) * LOG2E;
    u32x4 q[NM];
    {
        const char *qr = static_cast<const char *>(a.q) +
                         ((int64_t)(t.first + token) * a.q_stride + (int64_t)head * D + h * 8) * 2;
#pragma unroll
        for (int i = 0; i < NM; ++i) q[i] = u32x4{0, 0, 0, 0};
        if (live) {
#pragma unroll
            for (int i = 0; i < NM; ++i) q[i] = *reinterpret_cast<const u32x4 *>(qr + i * 32);
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    f32x16 o[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.0f;
    float m = NEG_INF, l = 0.0f;

    const int flip = lane ^ (lane >> 4 & 1);  // (see prefill_tile.h: value pieces without bank conflicts)
    // The wave's four pieces of a stage; past the end the last stage again, which nothing reads.
    auto load = [&](int stage, char *to) __attribute__((always_inline)) {
        stage = min(stage, last - 1);
        if (stage >= ids_from + ENTRIES) {  // uniform
            load_ids(stage);
            check_ids();
        }
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int unit = wave * UNITS + i, sub = unit % PER_PAGE;
            const int id = __builtin_amdgcn_readlane(ids, (stage - ids_from) * PAGES + unit / PER_PAGE);
            const int64_t at = (id < 0 ? 0 : base + id) * c.block_bytes + (int64_t)kvhead * PB + sub * 1024;
            ring_load(c.k + at + (uint32_t)lane * 16u, to + unit * 1024);
            ring_load(c.v + at + (uint32_t)flip * 16u, to + V + unit * 1024);
        }
    };
    // bit p: page p of the stage has no block (asked before the entries move on)
    auto holes_of = [&](int stage) {
        return (uint32_t)(__ballot(ids < 0) >> ((stage - ids_from) * PAGES)) & ((1u << PAGES) - 1);
    };

    if (first < last) {
        check_ids();
        uint32_t holes[STAGES];  // of the stages on their way
        holes[0] = holes_of(first);
        load(first, r0);
        holes[1] = holes_of(min(first + 1, last - 1));
        load(first + 1, r1);
        holes[2] = holes_of(min(first + 2, last - 1));
        load(first + 2, r2);
        holes[3] = 0;
        if (a.scale <= 0.0f) {  // a negative scale is the query's sign, a scale of zero a query of zeros
            const uint32_t sign = a.scale < 0.0f ? 0x80008000u : 0u, keep = a.scale == 0.0f ? 0u : ~0u;
#pragma unroll
            for (int i = 0; i < NM; ++i) q[i] = (q[i] ^ sign) & keep;
        }
        if (a.window > 0 || s1 * KEYS > tree0) {  // uniform
            fill_masks<NW>(c, a, t, parent, masks);
            if (a.window > 0 && pos >= 0) lo = max(0, t.pos0 + masks.count[pos - t.pos0] - a.window);
        }
        const int kfrag = (n >> 4) * PB + h * 256 + (n & 15) * 16, vfrag = ((n * 2 + h) ^ (n >> 3 & 1)) * 16;
        int stage = first;
        // A stage: its keys are at k; the ones three stages ahead go to where the last one was.
        auto body = [&](char *k, char *next, int at) __attribute__((always_inline)) {
            ring_barrier<2 * UNITS * (STAGES - 2)>();
            char *const v = k + V;
            const uint32_t missing = holes[at];
            {
                const int ahead = min(stage + STAGES - 1, last - 1);
                load(ahead, next);
                holes[(at + STAGES - 1) % STAGES] = holes_of(ahead);
            }
            const int t0 = stage * SK;
            if (missing || t0 + SK > t.len) {  // uniform
                // zeros in the values of keys past the end or without a block: they may be NaN
                for (int i = threadIdx.x; i < PAGES * PB / 16; i += NW * SAE_WAVE) {
                    const int p = i / (PB / 16), piece = i % 64 ^ (i >> 4 & 1);
                    u32x4 w = *reinterpret_cast<u32x4 *>(v + i * 16);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {  // token j of the piece's 8
                        const int key = t0 + p * SAE_KV_BLOCK + (piece & 1) * 4 + (j >> 2) * 8 + (j & 3);
                        if (key >= t.len || (missing >> p & 1)) w[j / 2] &= j & 1 ? 0xFFFFu : 0xFFFF0000u;
                    }
                    *reinterpret_cast<u32x4 *>(v + i * 16) = w;
                }
                ring_barrier<2 * UNITS * (STAGES - 1)>();
            }
            if (wrow < t.rows) {  // uniform: a wave without rows only moves its share
                f32x16 s[KT];
                const char *kp = k + kfrag, *vp = v + vfrag;
                // all of a stage's keys, and its values while the weights are computed
                u32x4 kf[NM * KT], vf[PAGES * NB];
#pragma unroll
                for (int i = 0; i < NM * KT; ++i) kf[i] = *reinterpret_cast<const u32x4 *>(kp + i % KT * 2 * PB + i / KT * 512);
#pragma unroll
                for (int u = 0; u < KT; ++u)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[u][i] = 0.0f;
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < NM * KT; ++i) s[i % KT] = mfma32<F16>(kf[i], q[i / KT], s[i % KT]);
#pragma unroll
                for (int i = 0; i < PAGES * NB; ++i) vf[i] = *reinterpret_cast<const u32x4 *>(vp + i / NB * PB + i % NB * 1024);
                __builtin_amdgcn_sched_barrier(0);
                if (missing || t0 < all0 || t0 + SK > all1) {  // uniform: not all is seen by all
                    asm volatile("");
#pragma unroll
                    for (int u = 0; u < KT; ++u) {
                        // bit b: the row sees key from0 + b
                        const int from0 = t0 + u * 32, from = min(max(lo - from0, 0), 32), to = min(max(tree0 - from0, 0), 32);
                        uint32_t seen = (uint32_t)((1ull << to) - 1) & ~(uint32_t)((1ull << from) - 1);
                        if (from0 + 32 > tree0 && pos >= 0) {
                            const int i0 = from0 - t.pos0, w = i0 >> 5;  // token of bit 0, maybe one before the first
                            const uint32_t *bits = masks.seen[pos - t.pos0];
                            const uint32_t y0 = w >= 0 && w < MASK_WORDS ? bits[w] : 0u, y1 = w >= -1 && w < MASK_WORDS - 1 ? bits[w + 1] : 0u;
                            seen |= (uint32_t)(((uint64_t)y1 << 32 | y0) >> (i0 & 31));
                        }
                        seen &= (missing >> (2 * u) & 1 ? 0u : 0xFFFFu) | (missing >> (2 * u + 1) & 1 ? 0u : 0xFFFF0000u);
                        seen >>= h * 4;
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (!(seen >> (i / 4 * 8 + i % 4) & 1)) s[u][i] = NEG_INF;
                    }
                }
                float top = s[0][0];
#pragma unroll
                for (int u = 0; u < KT; ++u)
#pragma unroll
                    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[u][i]);
                top = reference<F16>(max_halves(top) * sl, BIAS<F16>);
                if (__any(top > m + SLACK<F16>)) {
                    const float mn = fmaxf(m, top), f = mn == NEG_INF ? 0.0f : exp2_(m - mn);
                    m = mn;
                    l *= f;
#pragma unroll
                    for (int b = 0; b < NB; ++b) o[b] *= f;
                }
                const float mu = m == NEG_INF ? 0.0f : -m;
                u32x4 w[PAGES];
#pragma unroll
                for (int u = 0; u < KT; ++u)
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const float x = exp2_(__builtin_fmaf(s[u][i], sl, mu)), y = exp2_(__builtin_fmaf(s[u][i + 1], sl, mu));
                        l += x;
                        l += y;
                        w[u * 2 + i / 8][i / 2 % 4] = pack2<F16>(x, y);
                    }
#pragma unroll
                for (int i = 0; i < PAGES * NB; ++i) o[i % NB] = mfma32<F16>(vf[i], w[i / NB], o[i % NB]);
            }
            ++stage;
        };
#pragma unroll 1
        for (;;) {
            body(r0, r3, 0);
            if (stage >= last) break;
            body(r1, r0, 1);
            if (stage >= last) break;
            body(r2, r1, 2);
            if (stage >= last) break;
            body(r3, r2, 3);
            if (stage >= last) break;
        }
        ring_barrier<0>();  // what is on its way past the end arrives before the LDS is another's
    }
    finish<TYPE, D, NW, true>(c, a, plan, t, &masks, base, kvhead, wave, slot, nparts == 1, s0, s1, o, m, l);
}

template <int TYPE, int D>
hipError_t launch_ring(const KvDev &c, const AttnArgs &a, hipStream_t s)
{
    const Plan p = plan_of(c, a.heads, D, a.window, a.max_nodes);
    if (!p.groups) {
        hipLaunchKernelGGL((k_tree_ring<TYPE, D, false>), dim3(p.tiles * c.kvh), dim3(WAVES * SAE_WAVE), 0, s, c, a, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((k_tree_ring<TYPE, D, true>), dim3((unsigned)((p.groups + p.tiles) * c.kvh)), dim3(WAVES * SAE_WAVE), 0, s, c, a, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    return launch_tree_join<TYPE, D>(c, a, p, s);
}

template <int TYPE>
hipError_t launch_type(const KvDev &c, const AttnArgs &a, int dim, hipStream_t s)
{
    if constexpr (TYPE != SAE_KV_FP8)
        if (dim == 64) return launch_ring<TYPE, 64>(c, a, s);
    return launch_dim<TYPE, true>(c, a, dim, s);
}

}  // namespace

hipError_t launch_tree(const KvDev &c, const AttnArgs &a, int type, int dim, hipStream_t s)
{
    if (type == SAE_KV_BF16) return launch_type<SAE_KV_BF16>(c, a, dim, s);
    if (type == SAE_KV_F16) return launch_type<SAE_KV_F16>(c, a, dim, s);
    return launch_type<SAE_KV_FP8>(c, a, dim, s);
}
