// Causal attention of sequences' new tokens over the paged key-value cache.
//
// The query rows of a sequence and key-value head are its new tokens times the
// G query heads that share the head, row = token * G + head: keys and values are
// read once for all of them.  A workgroup takes a tile of 32 NW rows, a wave 32
// of them, over 64 keys (4 pages) a step, with the scores transposed:
//   S^T = K Q^T (64 keys x 32 rows), P = exp(S - m), O^T += V^T P^T
// on v_mfma_f32_32x32x16.  Keys and values of a step are staged in LDS, in the
// cache's own page layout, double-buffered: 16-bit pages go there directly from
// memory, an 8-bit cache through registers, widened to bf16 (times its scale) once
// for all waves.  Queries, scores, weights and outputs never leave registers:
// lane (n = lane % 32, h = lane / 32) holds all of row n's state (the other half
// of its keys and dimensions in lane n ^ 32), and the 16 scores a lane holds of 32
// keys are, rounded, the operand of the second product as they stand:
//   registers 8 u .. 8 u + 7 are tokens 4 h .. 4 h + 3 and 8 + 4 h .. of page u,
// which is the 16-byte piece h of a value page's dimension.
//
// Weights are rounded once to 16 bits for the second product (sums are of unrounded
// ones): a second number each, as decode takes, would make three products of two.  The
// error of the outputs is 1.3 to 1.4 times that of their own rounding.
//
// The running maximum is followed loosely: outputs are rescaled only when some
// row's maximum grew by more than 2^8, and weights are then 2^-8 .. 1 times what they are
// under the maximum itself (sums are fp32).  With f16 weights by more than 2^3.9, and
// weights are 2^12 times as large: they stay under 2^15.9 (the type ends at 2^16) and
// lose bits only below 2^-26 of the maximum that is followed, all below 2^-37.
//
// Bound by the matrix units and the power they may draw: 8,192 tokens behind 4,096
// cached ones, 32 heads of 128 on 8: 1,010 us, 1.09 PFLOP/s (a library product of
// 8,192^3 reaches 1.15 on the same card).  The products are under way 59 % of the
// time; the clock is 1.8 GHz then (2.0 GHz and 48 % before the loads went straight to
// LDS and a step's products shared their time with another's exponentials).  Products
// alone with five vector operations and two exponentials each reach 1.48 PFLOP/s.
//
// Where tiles are few, each one's keys are split over several workgroups, whose
// unnormalised outputs k_prefill_join adds in order.  Small calls are round trips and
// code: a launch fetches its code anew, and the kernel's size (40 KB, now 28) was 25 %
// of their time.  61 new tokens behind 1,440, 16 heads on 2: 13.6 + 5.2 us.
//
// TREE: the new tokens are a tree (k_tree.hip); beside the prefix a row sees its ancestors and itself.
#pragma once

#include <algorithm>

#include "attn_tile.h"

namespace {

using namespace attn;

constexpr int ROWS = 32;   // rows of a wave
// Keys of a step: 64, or 32 where a row's state and a step's scores would not fit
// the registers together.
constexpr int keys_of(int dim) { return dim == 256 ? 32 : 64; }
// Keys of a split at least (drawn calls, geometric means of four times 16: 128 37.6 /
// 45.1 / 23.4 / 29.2 us, 192 36.3 / 46.2 / 23.7 / 29.4, 256 37.5 / 46.2 / 23.5 / 29.0, 384
// 36.3 / 47.3 / 24.3 / 29.0).
constexpr int MIN_SPLIT = 192;
// Workgroups wanted: two per compute unit, one of the larger heads.
constexpr int groups_of(int dim) { return dim == 256 ? 256 : 512; }
// Keys of a table whose sequences are not split: no second launch (256: 49.3 / 60.0 / 29.8
// / 36.4 us, 512: 48.8 / 59.4 / 29.7 / 35.4, 1,024: 49.9 / 65.8 / 31.1 / 35.0).
constexpr int SHORT = 512;
// Of the running maximum, in powers of two; and how far under it the reference of the
// weights is.  bf16: above it, weights never pass 1 and outputs overflow no earlier than
// their sums do.  f16: a smaller slack rescales more often, most at heads of 256 (16
// ragged prompts / the long one; weights not biased, SLACK 8: 172 / 1,125 us; 5.9 and 10: 179
// / 1,143; 3.9 and 12: 190 / 1,178; 2.9 and 13: 203 / 1,206; heads of 128: 402 us for the
// long contexts, so 405).
template <bool F16>
constexpr float SLACK = F16 ? 3.9f : 8.0f;
template <bool F16>
constexpr float BIAS = F16 ? 12.0f : -8.0f;

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
    int tiles;   // row tiles of a head (an upper bound)
    int groups;  // workgroups per key-value head that fill the GPU, over which long tiles'
                 // keys are split; 0: none is
    int most;    // parts of a tile at most (from the keys that the table holds)
    int slots;   // parts that the workspace holds
    int joins;   // a tree's call: split tiles at most
};

// The rows of a workgroup and the keys they see.
struct Tile {
    int seq, first;        // first row of the sequence in the call's arrays
    int token0, head0;     // first row of the tile: token0 * G + head0
    int rows;              // rows of the tile that there are; 0: no such tile
    int pos0;              // position of the sequence's first new token (may be negative)
    int len;
    int step0, steps;      // steps of keys_of(dim) keys the tile sees: step0 .. step0 + steps - 1
    int tokens;            // of the sequence
};

// Tile `sub` of sequence seq.  (A call has fewer than 2^30 rows of a head: 32 bits.)
template <bool TREE>
__device__ __forceinline__ Tile tile_of(const KvDev &c, const AttnArgs &a, int seq, int sub, int rows, int keys)
{
    int first, tokens;
    kv::seq_rows(c, seq, first, tokens);
    const int len = kv::seq_len(c, seq), G = a.heads / c.kvh;
    Tile t = {seq, first, 0, 0, 0, len - tokens, len, 0, 0, tokens};
    const int row0 = sub * rows, end = tokens * G;
    if (sub < 0 || row0 >= end) return t;
    t.rows = min(rows, end - row0);
    t.token0 = (int)((uint32_t)row0 / (uint32_t)G);
    t.head0 = row0 - t.token0 * G;
    const int p0 = t.pos0 + t.token0, p1 = p0 + (t.head0 + t.rows - 1) / G;  // first and last position
    if (p1 >= 0 && !(TREE && tokens > a.max_nodes)) {
        // (a tree's rows may all be at its root's position)
        t.step0 = (a.window > 0 ? max(0, (TREE ? t.pos0 : p0) - a.window + 1) : 0) / keys;
        t.steps = p1 / keys + 1 - t.step0;
    }
    return t;
}

// Without split tiles: tile number `tile` of the call, sequences' tiles counted from
// q_start[r] G / rows + r on (at least what the sequences before have).
template <bool TREE>
__device__ __forceinline__ Tile find_tile(const KvDev &c, const AttnArgs &a, int tile, int rows, int keys)
{
    const int G = a.heads / c.kvh;
    if (!c.qs) {
        const int of_seq = (G + rows - 1) / rows;
        return tile_of<TREE>(c, a, tile / of_seq, tile % of_seq, rows, keys);
    }
    auto before = [&](int r) { return (int)((uint32_t)(min(max(c.qs[r], 0), c.n_tokens) * G) / (uint32_t)rows) + r; };
    int lo = 0, n = c.n_seq;
    while (n > 1) {  // 64 probes a round trip
        const int step = (n + SAE_WAVE - 1) / SAE_WAVE, r = lo + (int)__lane_id() * step;
        const bool below = r < lo + n && before(r) <= tile;
        const uint64_t m = __ballot(below);
        const int last = m ? 63 - __clzll((long long)m) : 0, end = lo + n;
        lo += last * step;
        n = min(step, end - lo);
    }
    lo = uniform(lo);
    return tile_of<TREE>(c, a, lo, tile - before(lo), rows, keys);
}

// With split tiles: every tile of a sequence in as many parts as its length calls for,
// so that a part has about the average work of a workgroup.  Workgroup x of a head
// takes part `part` of `parts` of tile `sub` of sequence `seq`.
struct Part {
    int seq, part, parts;  // seq < 0: none
    int sub;
    int slot;  // the part's place in the workspace, -1 for none
    // trees: the tile's number among those that are split, for its first part to note (-1: not this one), and
    // a number that no tile has, for this workgroup to say so
    int entry, clear;
};
constexpr int PER_THREAD = 2;  // sequences of a thread at most: plan_of() splits nothing of a call with more than 512

template <int NW>
__device__ __forceinline__ Part find_part(const KvDev &c, const AttnArgs &a, const Plan &plan, int x, int rows, int keys)
{
    __shared__ long long tmp[2][NW], found_rest;
    __shared__ int found_seq, found_parts;
    const int G = a.heads / c.kvh, chunk = (c.n_seq + NW * SAE_WAVE - 1) / (NW * SAE_WAVE);
    // tiles of sequence r, and the mean of their steps, about
    auto size = [&](int r, int &tiles, int &steps) {
        int first, tokens;
        kv::seq_rows(c, r, first, tokens);
        const int len = kv::seq_len(c, r);
        tiles = (int)((uint32_t)(tokens * G + rows - 1) / (uint32_t)rows);
        steps = (a.window > 0 ? min(a.window, len) : max(len - tokens / 2, 0)) / keys + 1;
    };
    auto share_of = [&](long long total) {
        return (int)max((total + plan.groups - 1) / plan.groups, (long long)(MIN_SPLIT / keys));
    };
    if (c.n_seq == 1) {  // uniform: no scans
        int tiles, steps;
        size(0, tiles, steps);
        const int parts = min(max(steps / share_of((long long)tiles * steps), 1), plan.most);
        return {x < (long long)tiles * parts ? 0 : -1, x % parts, parts, x / parts, x, -1, -1};
    }
    const int r0 = min((int)threadIdx.x * chunk, c.n_seq);
    int tiles[PER_THREAD], steps[PER_THREAD];
    long long work = 0;
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) {
        tiles[i] = steps[i] = 0;
        if (i < chunk && r0 + i < c.n_seq) {
            size(r0 + i, tiles[i], steps[i]);
            work += (long long)tiles[i] * steps[i];
        }
    }
    long long total;
    scan<NW>(work, total, tmp[0]);
    const int share = share_of(total);
    long long count = 0;
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) {
        steps[i] = min(max(steps[i] / share, 1), plan.most);  // parts from here on
        count += (long long)tiles[i] * steps[i];
    }
    long long before = scan<NW>(count, total, tmp[1]);
    if (x >= before && x < before + count) {  // one thread
#pragma unroll
        for (int i = 0; i < PER_THREAD; ++i) {
            const long long k = (long long)tiles[i] * steps[i];
            if (x >= before && x < before + k) {
                found_seq = r0 + i;
                found_parts = steps[i];
                found_rest = x - before;
            }
            before += k;
        }
    }
    __syncthreads();
    if (x >= total) return {-1, 0, 1, 0, x, -1, -1};
    const int parts = uniform(found_parts), rest = uniform((int)found_rest);
    return {uniform(found_seq), rest % parts, parts, rest / parts, x, -1, -1};
}

// A tree's call may have many more tiles than workgroups are wanted: parts are numbered in the
// workspace among those of split tiles alone, and so are these.  (Such a tile's keys are 3/2 shares at least and its parts at
// most 4/3 as many as shares: 4/3 groups in all, of the 2 groups that there are.)
template <int NW>
__device__ __forceinline__ Part find_part_tree(const KvDev &c, const AttnArgs &a, const Plan &plan, int x, int rows, int keys)
{
    __shared__ u64 sums[2][NW], found;
    __shared__ int found_seq, found_rest, found_parts;
    const int G = a.heads / c.kvh, chunk = (c.n_seq + NW * SAE_WAVE - 1) / (NW * SAE_WAVE);
    const int lane = (int)__lane_id(), wave = threadIdx.x / SAE_WAVE;
    // tiles of sequence r, and their steps
    auto size = [&](int r, int &tiles, int &steps) {
        int first, tokens;
        kv::seq_rows(c, r, first, tokens);
        const int len = kv::seq_len(c, r);
        tiles = (int)((uint32_t)(tokens * G + rows - 1) / (uint32_t)rows);
        steps = (a.window > 0 ? min(a.window + tokens, len) : len) / keys + 1;
        if (tokens > a.max_nodes) steps = 0;  // its rows see nothing; the join looks at no more than max_nodes' rows
    };
    // (in floating point: a quotient of 64-bit numbers is some hundred instructions; at least the quotient)
    auto parts_of = [&](u64 total, int steps) {
        const int share = max((int)fmin((double)total / plan.groups, 0x1p30) + 1, MIN_SPLIT / keys);  // (more than any tile's steps)
        return min(max((int)((uint32_t)(steps + share / 2) / (uint32_t)share), 1), plan.most);
    };
    if (c.n_seq == 1) {  // uniform
        int tiles, steps;
        size(0, tiles, steps);
        const int parts = parts_of((u64)tiles * steps, steps), sub = (int)((uint32_t)x / (uint32_t)parts);
        const bool held = sub < tiles && parts > 1;
        return {sub < tiles ? 0 : -1, x - sub * parts, parts, sub, held ? x : -1, held && x == sub * parts ? sub : -1,
                x >= (parts > 1 ? tiles : 0) ? x : -1};
    }
    const int r0 = min((int)threadIdx.x * chunk, c.n_seq);
    int tiles[PER_THREAD], steps[PER_THREAD];
    u64 work = 0;
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) {
        tiles[i] = steps[i] = 0;
        if (i < chunk && r0 + i < c.n_seq) {
            size(r0 + i, tiles[i], steps[i]);
            work += (u64)tiles[i] * steps[i];
        }
    }
    work = sum_upto(work);
    if (lane == SAE_WAVE - 1) sums[0][wave] = work;
    __syncthreads();
    u64 total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) total += sums[0][w];
    // three sums in one: workgroups (44 bits), split tiles (10), their parts (10).  No q_start passes them: rows counted again for
    // several sequences are 512 times 2^23 tiles at most, and 2/3 and 4/3 of 512 groups bound the others whatever is summed.
    auto packed = [](u64 tiles, u64 parts) { return tiles * parts << 20 | (parts > 1 ? tiles << 10 | tiles * parts : 0); };
    u64 count = 0;
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) {
        steps[i] = parts_of(total, steps[i]);  // parts from here on
        count += packed(tiles[i], steps[i]);
    }
    const u64 upto_here = sum_upto(count);
    if (lane == SAE_WAVE - 1) sums[1][wave] = upto_here;
    __syncthreads();
    u64 before = upto_here - count, all = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        before += w < wave ? sums[1][w] : 0;
        all += sums[1][w];
    }
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) {
        const long long rest = x - (long long)(before >> 20);
        if (rest >= 0 && rest < tiles[i] * steps[i]) {  // one thread
            found_seq = r0 + i;
            found_rest = (int)rest;
            found_parts = steps[i];
            found = before;
        }
        before += packed(tiles[i], steps[i]);
    }
    __syncthreads();
    // A q_start that decreases may call for more workgroups than the grid has, a split tile's first one among them: no tile is
    // noted then, or the join would go by an entry that nobody wrote.
    const bool over = all >> 20 > (u64)(plan.groups + plan.tiles);
    const int clear = over || x >= (int)(all >> 10 & 0x3FF) ? x : -1;
    if (x >= (long long)(all >> 20)) return {-1, 0, 1, 0, -1, -1, clear};
    const int parts = uniform(found_parts), rest = uniform(found_rest), sub = (int)((uint32_t)rest / (uint32_t)parts);
    const u64 at = (u64)uniform((long long)found);
    return {uniform(found_seq), rest - sub * parts, parts, sub, parts > 1 ? (int)(at & 0x3FF) + rest : -1,
            !over && parts > 1 && rest == sub * parts ? (int)(at >> 10 & 0x3FF) + sub : -1, clear};
}

// A split tile as the workspace has it, by the workgroup of its first part.
struct Split {
    int token, head0, rows;  // token: row of the call's arrays of its first token
    int parts;               // in workgroups x .. x + parts - 1; < 2: none
};
// The same for a tree's call, whose split tiles and their parts are numbered by themselves.
struct TreeSplit {
    int token;
    int shape;  // head0 | rows << 16
    int slot;   // the first part's place in the workspace, the others behind it
    int parts;  // < 2: none
};
static_assert(sizeof(TreeSplit) == sizeof(Split), "they take the same room");

// What a workgroup of a tree's call notes of its part for the join.
__device__ __forceinline__ void note_split(const AttnArgs &a, const Plan &plan, const Part &p, const Tile &t, int kvhead)
{
    if (kvhead != 0 || threadIdx.x != 0) return;
    TreeSplit *const at = static_cast<TreeSplit *>(a.work);
    // (no place is written past the last)
    if (p.clear >= 0 && p.clear < plan.joins) at[p.clear] = TreeSplit{0, 0, 0, 0};
    if (p.entry >= 0 && p.entry < plan.joins)
        at[p.entry] = TreeSplit{t.first + t.token0, t.head0 | t.rows << 16, p.slot, p.slot + p.parts <= plan.slots ? p.parts : 0};
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

// Whether any value of keys from .. to - 1 is not finite: the whole wave, a page at a time.
// (An 8-bit value may also pass the range of bf16 with its scale.)
template <int TYPE, int D>
__device__ __forceinline__ bool any_odd(const KvDev &c, const Tile &t, int64_t base, int kvhead, int from, int to)
{
    constexpr bool FP8 = TYPE == SAE_KV_FP8;
    constexpr int E = FP8 ? 1 : 2, PAGE = SAE_KV_BLOCK * D * E;
    constexpr uint32_t INF = FP8 ? 0x7Fu : is_f16(TYPE) ? 0x7C00u : 0x7F80u;  // the bits that say it
    const int lane = (int)__lane_id();
    bool odd = false;
#pragma unroll 1
    for (int page = from / SAE_KV_BLOCK; page * SAE_KV_BLOCK < to; ++page) {
        const int id = c.ids[(int64_t)t.seq * c.max_blocks + page], lo = from - page * SAE_KV_BLOCK, hi = to - page * SAE_KV_BLOCK;
        if (base < 0 || id < 0 || id >= c.bpi) continue;  // uniform
        const char *vp = c.v + (base + id) * c.block_bytes + (int64_t)kvhead * PAGE;
#pragma unroll 1
        for (int i = lane; i < PAGE / 16; i += SAE_WAVE) {
            const u32x4 w = *reinterpret_cast<const u32x4 *>(vp + i * 16);
#pragma unroll
            for (int j = 0; j < 16 / E; ++j) {
                const int token = (i & 1) * 4 + (j >> 2 & 1) * 8 + (j & 3);
                odd |= token >= lo && token < hi && (w[j * E / 4] >> (8 * E * (j % (4 / E))) & INF) == INF;
            }
        }
        if constexpr (FP8) {
            const int token = lane & 15;
            odd |= token >= lo && token < hi && c.vs[(base + id) * c.scale_stride + kvhead * SAE_KV_BLOCK + token] >= 240;
        }
    }
    return __any(odd);
}

// A sequence's drafted tokens (a tree, at most MAX_NODES of them): bit i of row j says that token j
// sees token i, itself or an ancestor of it that the window reaches.
constexpr int MAX_NODES = SAE_TREE_MAX, MASK_WORDS = MAX_NODES / 32;
struct Masks {
    uint32_t seen[MAX_NODES][MASK_WORDS + 1];  // (an odd row: lanes read all banks)
    int up[MAX_NODES];     // a token's ancestor 2^k above, -1 for none
    int count[MAX_NODES];  // tokens on the way there; at the end 1 + the token's depth
};

// Fills `m`, a token a thread.  After round k a token's row holds itself and its next
// 2^k - 1 ancestors: log2(tokens) rounds, whatever the tree's depth.  A window of H is the binary
// digits of H as such pieces, one behind the other.
template <int NW>
__device__ __forceinline__ void fill_masks(const KvDev &c, const AttnArgs &a, const Tile &t, int parent, Masks &m)
{
    static_assert(NW * SAE_WAVE == MAX_NODES, "a thread for each token");
    const int n = t.tokens, j = threadIdx.x, words = (n + 31) / 32;
    const int hops = a.window > 0 ? min(a.window, n) : 0;
    const bool live = j < n;
    if (live && (parent < -1 || parent >= j)) {
        if (c.status) atomicOr(c.status, (uint32_t)SAE_ST_BAD_TREE);
        parent = -1;
    }
    if (n <= SAE_WAVE) {  // uniform: a wave by itself, its lanes' rows in registers
        if (threadIdx.x < SAE_WAVE) {
            u64 row = live ? 1ull << j : 0, near = 0;
            int up = live ? parent : -1, count = 1, at = live ? j : -1;
#pragma unroll 1
            for (int k = 0;; ++k) {
                if (hops >> k & 1) {  // uniform
                    const u64 more = __shfl(row, max(at, 0));
                    const int next = __shfl(up, max(at, 0));
                    near |= at >= 0 ? more : 0;
                    at = at >= 0 ? next : -1;
                }
                if (1 << k >= n) break;
                const u64 more = __shfl(row, max(up, 0));
                const int next = __shfl(up, max(up, 0)), tokens = __shfl(count, max(up, 0));
                row |= up >= 0 ? more : 0;
                count += up >= 0 ? tokens : 0;
                up = up >= 0 ? next : -1;
            }
            if (hops) row = near;
            m.seen[j][0] = (uint32_t)row;
            m.seen[j][1] = (uint32_t)(row >> 32);
#pragma unroll
            for (int w = 2; w < MASK_WORDS; ++w) m.seen[j][w] = 0;
            m.count[j] = count;
        }
        __syncthreads();
        return;
    }
    uint32_t row[MASK_WORDS], near[MASK_WORDS];
#pragma unroll
    for (int w = 0; w < MASK_WORDS; ++w) {
        row[w] = live && w == j / 32 ? 1u << (j % 32) : 0u;
        near[w] = 0;
    }
    int up = live ? parent : -1, count = 1, at = live ? j : -1;
#pragma unroll
    for (int w = 0; w < MASK_WORDS; ++w) m.seen[j][w] = row[w];
    m.up[j] = up;
    m.count[j] = count;
    __syncthreads();
#pragma unroll 1
    for (int k = 0;; ++k) {
        if ((hops >> k & 1) && at >= 0) {
#pragma unroll
            for (int w = 0; w < MASK_WORDS; ++w)
                if (w < words) near[w] |= m.seen[at][w];
            at = m.up[at];
        }
        if (1 << k >= n) break;  // uniform
        if (up >= 0) {
#pragma unroll
            for (int w = 0; w < MASK_WORDS; ++w)
                if (w < words) row[w] |= m.seen[up][w];
            count += m.count[up];
            up = m.up[up];
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < MASK_WORDS; ++w)
            if (w < words) m.seen[j][w] = row[w];
        m.up[j] = up;
        m.count[j] = count;
        __syncthreads();
    }
    if (hops) {
        __syncthreads();  // the last pieces have been read
#pragma unroll
        for (int w = 0; w < MASK_WORDS; ++w) m.seen[j][w] = near[w];
        __syncthreads();
    }
}

// The wave's rows over keys key0 .. key1 - 1 once more, one key at a time on the
// vector units, each row adding the keys it sees and no other: the slow path
// for values that are not finite and that not all of the rows see, and for scores past
// 2^24 (about 130 times as long as the loop it replaces, with the same state after it).
template <int TYPE, int D, bool TREE>
__device__ void redo(const KvDev &c, const AttnArgs &a, const Tile &t, const Masks *masks, int64_t base, int kvhead, int key0,
                     int key1, int token, int head, int pos, f32x16 (&o)[D / 32], float &m, float &l)
{
    constexpr bool FP8 = TYPE == SAE_KV_FP8, F16 = is_f16(TYPE);
    constexpr int E = FP8 ? 1 : 2, PAGE = SAE_KV_BLOCK * D * E, ND = FP8 ? 2 : 1;
    const int h = (int)__lane_id() >> 5;
    const int lo = a.window > 0 ? max(0, (TREE ? t.pos0 + masks->count[token] - 1 : pos) - a.window + 1) : 0;
    const uint16_t *q = static_cast<const uint16_t *>(a.q) + (int64_t)(t.first + token) * a.q_stride + (int64_t)head * D;
    m = NEG_INF;
    l = 0.0f;
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.0f;
#pragma unroll 1
    for (int key = key0; key < key1; ++key) {
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
        if (TREE && key >= t.pos0) {
            if (key > pos || !(masks->seen[token][(key - t.pos0) / 32] >> ((key - t.pos0) % 32) & 1)) continue;
        } else if (key < lo || key > pos) continue;
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

// The workspace: plan.slots descriptions, then per slot, head and wave a part's outputs, maxima and sums as the lanes
// hold them.  Prefill: a slot and a Split for each of workgroups 0 .. groups + tiles - 1.  Trees: a slot for each part of a
// split tile, and the first plan.joins descriptions are the split tiles' TreeSplits.
__device__ __forceinline__ float *parts_of(const AttnArgs &a, const Plan &plan)
{
    return reinterpret_cast<float *>(static_cast<Split *>(a.work) + plan.slots);
}
__host__ __device__ constexpr int64_t part_floats(int dim) { return ROWS * (dim + 4); }
template <int D, int NW>
__device__ __forceinline__ int64_t part_at(const KvDev &c, int64_t x, int kvhead, int wave)
{
    return ((x * c.kvh + kvhead) * NW + wave) * part_floats(D);
}

// An output, which is a mean of values: finite f16 ones have none past their largest, where
// the weights' rounding could take it (to infinity).
template <bool F16>
__device__ __forceinline__ float mean(float x)
{
    if constexpr (F16) return fabsf(x) < __builtin_inff() ? __builtin_amdgcn_fmed3f(x, -65504.0f, 65504.0f) : x;
    else return x;
}

// The end of a tile's part: outputs where it is the only one.
template <int TYPE, int D, int NW, bool TREE>
__device__ __forceinline__ void finish(const KvDev &c, const AttnArgs &a, const Plan &plan, const Tile &t, const Masks *masks,
                                       int64_t base, int kvhead, int wave, int x, bool whole, int s0, int s1, f32x16 (&o)[D / 32],
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
    // not see its key.  Only outputs can show that (weights are a row's own), and it is wrong
    // only where the key is not seen by all the wave's rows: keys before the last row's
    // window or past the first row's position.  (A prefix that every row sees may hold
    // anything: the call takes as long as ever.)
    bool odd = false;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd |= !(fabsf(o[b][i]) < __builtin_inff());
    // A weight's exponent is one fused product and difference, under a maximum that was
    // rounded: where fp32 holds scores to whole numbers or less, the rounding would be an
    // exponent that may be anything.  Such rows take the slow path as well.
    const bool huge = fabsf(m) >= 0x1p24f && fabsf(m) < __builtin_inff();
    if (__any(live && (huge || (odd && l < __builtin_inff())))) {
        const int k0 = s0 * keys_of(D), k1 = min(s1 * keys_of(D), t.len);
        // (a tree's tokens are not seen by all)
        const int p0 = TREE ? t.pos0 - 1 : t.pos0 + t.token0 + (t.head0 + wave * ROWS) / G;
        const int p1 = t.pos0 + t.token0 + (t.head0 + min(wave * ROWS + ROWS, t.rows) - 1) / G;
        if (__any(live && huge) || any_odd<TYPE, D>(c, t, base, kvhead, max(p0 + 1, k0), k1) ||
            (a.window > 0 && any_odd<TYPE, D>(c, t, base, kvhead, k0, min(p1 - a.window + 1, k1))))
            redo<TYPE, D, TREE>(c, a, t, masks, base, kvhead, k0, k1, token, head, live ? t.pos0 + token : -1, o, m, l);
    }

    l += __shfl_xor(l, 32);
    if (whole) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;  // no key seen, or every score -inf
        char *to = static_cast<char *>(a.out) + ((int64_t)(t.first + token) * a.out_stride + (int64_t)head * D + h * 8) * 2;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 8) {
                // The halves hold dimensions 0 .. 3 and 4 .. 7 of eight; they trade, and each has
                // eight in a row (stores of 8 bytes: 3 % more for drawn calls, 5 % for 16 prompts of 600).
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = pack2<F16>(mean<F16>(o[b][i + 2 * e] * inv), mean<F16>(o[b][i + 2 * e + 1] * inv));
                const auto x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
                const auto y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
                if (live) *reinterpret_cast<u32x4 *>(to + (b * 32 + i * 2) * 2) = u32x4{x[0], y[0], x[1], y[1]};
            }
        if (!live) return;
        if (a.lse && h == 0)
            a.lse[(int64_t)(t.first + token) * a.heads + head] = l == 0.0f ? NEG_INF : (m + log2_(l)) * LN2;
        return;
    }
    if (TREE && (x >= plan.slots || wave * ROWS >= t.rows)) return;  // uniform
    // a part: maxima, sums and outputs as the lanes hold them
    float *to = parts_of(a, plan) + part_at<D, NW>(c, x, kvhead, wave);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<f32x4 *>(to + (b * 4 + i) * 256 + lane * 4) =
                f32x4{o[b][i * 4], o[b][i * 4 + 1], o[b][i * 4 + 2], o[b][i * 4 + 3]};
    *reinterpret_cast<float2 *>(to + ROWS * D + lane * 2) = float2{m, l};
}

template <int TYPE, int D, int NW, bool SPLIT, bool TREE>
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
    Masks *masks = nullptr;
    if constexpr (TREE) {
        __shared__ Masks held;
        masks = &held;
    }

    // blocks go round-robin over the XCDs: the key-value head varies fastest, so
    // that the tiles that read the same keys tend to share an L2
    const int x = blockIdx.x / c.kvh, kvhead = blockIdx.x % c.kvh, G = a.heads / c.kvh;
    Tile t;
    int part = 0, nparts = 1, slot = x;
    if constexpr (SPLIT) {
        Part p;
        if constexpr (TREE) p = find_part_tree<NW>(c, a, plan, x, NW * ROWS, KEYS);
        else p = find_part<NW>(c, a, plan, x, NW * ROWS, KEYS);
        if (p.seq >= 0) t = tile_of<TREE>(c, a, p.seq, p.sub, NW * ROWS, KEYS);
        slot = p.slot;
        if constexpr (TREE) {
            note_split(a, plan, p, t, kvhead);
        } else if (kvhead == 0 && threadIdx.x == 0)
            // (parts past the grid: only with a q_start that decreases)
            static_cast<Split *>(a.work)[x] = p.seq >= 0 && p.part == 0 && x + p.parts <= plan.groups + plan.tiles
                                                  ? Split{t.first + t.token0, t.head0, t.rows, p.parts}
                                                  : Split{0, 0, 0, 0};
        if (p.seq < 0) return;
        part = p.part;
        nparts = p.parts;
    } else {  // long tiles (late ones of a prompt) come first
        t = find_tile<TREE>(c, a, plan.tiles - 1 - x, NW * ROWS, KEYS);
    }
    if (t.rows == 0) return;
    const int lane = (int)__lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / SAE_WAVE);
    const int n = lane & 31, h = lane >> 5;
    const int64_t base = kv::seq_base(c, t.seq);
    const int s0 = t.step0 + (int)((int64_t)t.steps * part / nparts);
    const int s1 = t.step0 + (int)((int64_t)t.steps * (part + 1) / nparts);
    int parent = -1;  // of the tree's token threadIdx.x
    if constexpr (TREE) {
        if (t.tokens > a.max_nodes && threadIdx.x == 0 && c.status) atomicOr(c.status, (uint32_t)SAE_ST_BAD_TREE);
        if (t.tokens <= a.max_nodes && (int)threadIdx.x < t.tokens) parent = a.parent[t.first + threadIdx.x];
    }

    // this lane's row
    const int wrow = wave * ROWS, row = wrow + n;
    const bool live = row < t.rows;
    const int pos = live ? t.pos0 + t.token0 + (t.head0 + row) / G : -1;  // keys lo .. pos are seen
    // a row that sees nothing: a first key past all others
    int lo = pos < 0 ? 1 << 30 : a.window > 0 ? max(0, pos - a.window + 1) : 0;
    // the first of a tree's tokens; keys before it are seen from lo on
    const int tree0 = TREE ? max(t.pos0, 0) : 0;
    const uint32_t span = pos < 0 ? 0u : (uint32_t)(pos - lo);
    // the wave's first and last position (rows are in order of position)
    const bool full_rows = wrow + ROWS <= t.rows;
    const int wp0 = wrow < t.rows ? t.pos0 + t.token0 + (t.head0 + wrow) / G : -1;
    const int wp1 = wrow < t.rows ? t.pos0 + t.token0 + (t.head0 + min(wrow + ROWS, t.rows) - 1) / G : -1;
    const int wlo1 = a.window > 0 ? max(0, wp1 - a.window + 1) : 0;  // the last row's first key

    // table entries of 16 steps: lane 4 j + p has page p of step ids_from + j, -1 for none
    int ids = -1, ids_from = 0;
    auto load_ids = [&](int step) __attribute__((always_inline)) {
        ids_from = step;
        const int page = step * PAGES + lane;
        ids = -1;
        if (page * SAE_KV_BLOCK < t.len && step + lane / PAGES < s1) ids = c.ids[(int64_t)t.seq * c.max_blocks + page];
    };
    auto check_ids = [&]() __attribute__((always_inline)) {
        if (ids >= c.bpi) kv::report(c);
        if (base < 0 || ids >= c.bpi) ids = -1;
    };
    auto fetch_ids = [&](int step) {
        load_ids(step);
        check_ids();
    };
    // The first table entries before the queries: the keys wait for them alone, and loads
    // arrive in order (queries first: 5.5 us from here to the first keys, now 3.5; sixteen
    // prompts of 600 tokens 98 us, now 93).
    load_ids(s0);
    __builtin_amdgcn_sched_barrier(0);
    const float sl = a.scale == 0.0f ? 1.0f : fabsf(a.scale) * LOG2E;
    u32x4 q[NM];
    {
        const int token = live ? t.token0 + (t.head0 + row) / G : 0, head = kvhead * G + (live ? (t.head0 + row) % G : 0);
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
    float m = NEG_INF, l = 0.0f;  // m: the reference of weights

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
    // Unit i of a stage widened to bf16 (times its tokens' scales) and stored.
    auto store_k1 = [&](const St &st, char *lds, int i) __attribute__((always_inline)) {
        if constexpr (FP8) {  // 16 dimensions of token lane % 16
            const int unit = wave * St::UNITS + i, p = unit / St::PER_PAGE, sub = unit % St::PER_PAGE;
            char *to = lds + p * PB + (sub * 4 + (lane >> 4)) * 512 + (lane & 15) * 16;
            const float ks = scale_of(st.s[i][0], 0);
            *reinterpret_cast<u32x4 *>(to) = widen8(st.x[i][0], st.x[i][1], ks);
            *reinterpret_cast<u32x4 *>(to + 256) = widen8(st.x[i][2], st.x[i][3], ks);
        }
    };
    auto store_v1 = [&](const St &st, char *lds, int i) __attribute__((always_inline)) {
        if constexpr (FP8) {  // 8 tokens of two dimensions
            const int unit = wave * St::UNITS + i, p = unit / St::PER_PAGE, sub = unit % St::PER_PAGE;
            u32x4 w[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                // tokens 4 j .. 4 j + 3: a token's two dimensions side by side share a scale and one
                // conversion (each value by itself: 442 us for the long 8-bit prompts, so 423)
                const uint32_t x = st.x[i][j], y = st.x[i][2 + j], sc = st.s[i][j];
                const uint32_t a01 = __builtin_amdgcn_perm(y, x, 0x05010400u), a23 = __builtin_amdgcn_perm(y, x, 0x07030602u);
                const uint32_t t0 = widen2<false>(a01, scale_of(sc, 0)), t1 = widen2<true>(a01, scale_of(sc, 1));
                const uint32_t t2 = widen2<false>(a23, scale_of(sc, 2)), t3 = widen2<true>(a23, scale_of(sc, 3));
                w[0][j * 2] = __builtin_amdgcn_perm(t1, t0, 0x05040100u);
                w[1][j * 2] = __builtin_amdgcn_perm(t1, t0, 0x07060302u);
                w[0][j * 2 + 1] = __builtin_amdgcn_perm(t3, t2, 0x05040100u);
                w[1][j * 2 + 1] = __builtin_amdgcn_perm(t3, t2, 0x07060302u);
            }
            char *to = lds + p * PB + (sub * 2 + (lane >> 5)) * 1024 + (flip & 31) * 16;
            *reinterpret_cast<u32x4 *>(to) = w[0];
            *reinterpret_cast<u32x4 *>(to + 512) = w[1];
        }
    };
    auto store_k = [&](const St &st, char *lds) {
#pragma unroll
        for (int i = 0; i < St::UNITS; ++i) store_k1(st, lds, i);
    };
    auto store_v = [&](const St &st, char *lds) {
#pragma unroll
        for (int i = 0; i < St::UNITS; ++i) store_v1(st, lds, i);
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
        if (holes == 0 && full_rows && t0 + KEYS - 1 <= (TREE ? min(wp0, tree0 - 1) : wp0) && t0 >= wlo1) return;  // uniform
        asm volatile("");  // a branch: the comparisons are not worth taking on every step
        if constexpr (TREE) {
#pragma unroll
            for (int u = 0; u < KT; ++u) {
                // bit b: the row sees key k0 + b
                const int k0 = t0 + u * 32, from = min(max(lo - k0, 0), 32), to = min(max(tree0 - k0, 0), 32);
                uint32_t seen = (uint32_t)((1ull << to) - 1) & ~(uint32_t)((1ull << from) - 1);
                if (k0 + 32 > tree0 && pos >= 0) {
                    const int i0 = k0 - t.pos0, w = i0 >> 5;  // token of bit 0, maybe one before the first
                    const uint32_t *mine = masks->seen[pos - t.pos0];
                    const uint32_t x = w >= 0 && w < MASK_WORDS ? mine[w] : 0u, y = w >= -1 && w < MASK_WORDS - 1 ? mine[w + 1] : 0u;
                    seen |= (uint32_t)(((uint64_t)y << 32 | x) >> (i0 & 31));
                }
                seen >>= h * 4;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!(seen >> (i / 4 * 8 + i % 4) & 1)) s[u][i] = NEG_INF;
            }
        } else {
            const uint32_t rel = (uint32_t)(t0 + h * 4 - lo);  // lo <= key <= pos: key - lo, without sign, is at most span
#pragma unroll
            for (int u = 0; u < KT; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (rel + (uint32_t)(u * 32 + i / 4 * 8 + i % 4) > span) s[u][i] = NEG_INF;
        }
        if (holes) {
            asm volatile("");
#pragma unroll
            for (int p = 0; p < PAGES; ++p)
                if (holes >> p & 1) {
                    asm volatile("");
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[p / 2][p % 2 * 8 + i] = NEG_INF;
                }
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
        top = reference<F16>(top, BIAS<F16>);
        if (!__any(top > m + SLACK<F16>)) return;
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
    auto outputs = [&](const u32x4 (&w)[PAGES], const char *lds) {
        const char *vp = lds + vfrag;
#pragma unroll
        for (int p = 0; p < PAGES; ++p)
#pragma unroll
            for (int b = 0; b < NB; ++b)
                o[b] = mfma32<F16>(*reinterpret_cast<const u32x4 *>(vp + p * PB + b * 1024), w[p], o[b]);
    };

    if (TREE && s0 < s1 && wrow >= t.rows) {  // uniform: a wave without rows moves its share of keys and values
        St sk, sv;
        check_ids();
        uint32_t holes0 = holes_of(s0);
        const int next = min(s0 + 1, s1 - 1);
        {
            St k0;
            load_k(s0, k0, k_even);
            load_v(s0, sv, v_even);
            load_k(next, sk, k_odd);
            store_k(k0, k_even);
            store_v(sv, v_even);
            store_k(sk, k_odd);
        }
        uint32_t holes = holes_of(next);
        if (a.window > 0 || s1 * KEYS > tree0) fill_masks<NW>(c, a, t, parent, *masks);
        barrier();
        barrier();
        int step = s0;
        auto body = [&](int buf) __attribute__((always_inline)) {
            clean_v(step, holes0, lds_v[buf]);
            const int ahead = min(step + 2, s1 - 1);
            if (ahead >= ids_from + SAE_WAVE / PAGES) fetch_ids(step + 1);
            holes0 = holes;
            holes = holes_of(ahead);
            load_k(ahead, sk, lds_k[buf]);
            load_v(step + 1, sv, lds_v[buf ^ 1]);
            store_k(sk, lds_k[buf]);
            store_v(sv, lds_v[buf ^ 1]);
            barrier();
            ++step;
        };
        while (step + 1 < s1) {
            body(0);
            if (step + 1 >= s1) break;
            body(1);
        }
        clean_v(step, holes0, (step - s0) & 1 ? v_odd : v_even);
    } else if (s0 < s1) {
        // Step t's weights are computed while the matrix units take step t + 1's
        // scores, and that step's maximum while they add step t to the outputs: keys
        // are staged one step ahead of values.
        St sk, sv;
        f32x16 s[KT];
        u32x4 w[PAGES];
        check_ids();
        uint32_t holes0 = holes_of(s0), holes = 0;  // of the step whose values, and of the one whose scores come next
        {
            St k0;
            const int next = min(s0 + 1, s1 - 1);
            load_k(s0, k0, k_even);
            load_v(s0, sv, v_even);
            load_k(next, sk, k_odd);
            holes = holes_of(next);
            if (a.scale <= 0.0f) {  // a negative scale is the query's sign, a scale of zero a query of zeros
                const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u, keep = a.scale == 0.0f ? 0u : ~0u;
#pragma unroll
                for (int i = 0; i < NM; ++i) q[i] = (q[i] ^ flip) & keep;
            }
            store_k(k0, k_even);
            store_v(sv, v_even);
            store_k(sk, k_odd);
        }
        if constexpr (TREE) {
            // uniform: parts whose keys all rows see do not need it
            if (a.window > 0 || s1 * KEYS > tree0) {
                fill_masks<NW>(c, a, t, parent, *masks);
                if (a.window > 0 && pos >= 0) lo = max(0, t.pos0 + masks->count[pos - t.pos0] - a.window);
            }
        }
        barrier();
        scores(s, 0);
        barrier();  // every wave has read the first keys: the next loads go over them
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
                    // (beside the second half: behind them all, heads of 256 took 681 us where this takes 643)
                    if (FP8 && i >= N / 2 && (i - N / 2) * 2 * St::UNITS % (N / 2) == 0) {
                        const int u = (i - N / 2) * 2 * St::UNITS / (N / 2);
                        if (u < St::UNITS) store_k1(sk, lds_k[buf], u);
                        else store_v1(sv, lds_v[buf ^ 1], u - St::UNITS);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            follow(max_halves(top) * sl);
            holes0 = holes;
            holes = holes2;
            barrier();  // keys of step + 2 and values of step + 1 are whole, what they replaced was read before
            ++step;
        };
        f32x16 t[KT];
        while (step + 1 < s1) {  // two steps a round, each on its own buffers
            body(s, t, 0);
            if (step + 1 >= s1) break;
            body(t, s, 1);
        }
        // the last step: its scores are in t after an odd number of steps
        const bool odd = (step - s0) & 1;
        if (odd) {
#pragma unroll
            for (int u = 0; u < KT; ++u) s[u] = t[u];
        }
        char *const last = odd ? v_odd : v_even;
        clean_v(step, holes0, last);
        weights(s, w);
        outputs(w, last);
    }

    finish<TYPE, D, NW, TREE>(c, a, plan, t, masks, base, kvhead, wave, slot, nparts == 1, s0, s1, o, m, l);
}

// Adds a tile's parts, in order: lanes hold what they held in k_prefill, a wave
// one 32-dimension block of 32 rows.
template <int TYPE, int D, int NW>
__global__ void __launch_bounds__(NW * SAE_WAVE) k_prefill_join(KvDev c, AttnArgs a, Plan plan)
{
    constexpr bool F16 = is_f16(TYPE);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / SAE_WAVE), b = blockIdx.y;
    const int x = blockIdx.x / c.kvh, kvhead = blockIdx.x % c.kvh, G = a.heads / c.kvh;
    const Split t = static_cast<const Split *>(a.work)[x];
    if (t.parts < 2 || wave * ROWS >= t.rows) return;
    const int lane = (int)__lane_id(), n = lane & 31, h = lane >> 5;
    const int row = wave * ROWS + n;
    const float *from = parts_of(a, plan) + part_at<D, NW>(c, x, kvhead, wave);
    const int64_t stride = c.kvh * NW * part_floats(D);
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
    if (row >= t.rows) return;
    const int64_t token = t.token + (t.head0 + row) / G, head = kvhead * G + (t.head0 + row) % G;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    char *to = static_cast<char *>(a.out) + (token * a.out_stride + head * D + b * 32 + h * 4) * 2;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        *reinterpret_cast<u32x2 *>(to + i * 16) =
            u32x2{pack2<F16>(mean<F16>(o[i][0] * inv), mean<F16>(o[i][1] * inv)),
                  pack2<F16>(mean<F16>(o[i][2] * inv), mean<F16>(o[i][3] * inv))};
    if (a.lse && h == 0 && b == 0) a.lse[token * a.heads + head] = l == 0.0f ? NEG_INF : (m + log2_(l)) * LN2;
}

// 128 rows a workgroup.  256 rows (8 waves, one workgroup per compute unit) read half as
// much from L2: 990 us for the long prompt instead of 1,006, but 207 instead of 179
// for sixteen ragged ones.
constexpr int WAVES = 4;

// Adds a split tile's parts for a tree's call: a workgroup 32 dimensions of 32 rows, wave w parts
// w, w + 4, ..., four of them in flight.  (A wave for each 32 rows, one part after the other, as
// k_prefill_join: 14.7 us where 64 rows of each tile lie in 8 parts, 8.6 in 2 of 3.)
template <int TYPE, int D>
__global__ void __launch_bounds__(4 * SAE_WAVE) k_tree_join(KvDev c, AttnArgs a, Plan plan)
{
    constexpr int NW = 4, UN = 4;
    constexpr bool F16 = is_f16(TYPE);
    __shared__ f32x4 os[NW][4][SAE_WAVE];
    __shared__ float2 mls[NW][SAE_WAVE];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / SAE_WAVE), b = blockIdx.y, tile = blockIdx.z;
    const int kvhead = blockIdx.x % c.kvh, G = a.heads / c.kvh;
    const TreeSplit t = static_cast<const TreeSplit *>(a.work)[blockIdx.x / c.kvh];
    const int head0 = t.shape & 0xFFFF, rows = t.shape >> 16, slot = t.slot;
    if (t.parts < 2 || tile * ROWS >= rows) return;
    const int lane = (int)__lane_id(), n = lane & 31, h = lane >> 5;
    const int row = tile * ROWS + n;
    const float *from = parts_of(a, plan) + part_at<D, WAVES>(c, slot, kvhead, tile);
    const int64_t stride = c.kvh * WAVES * part_floats(D);
    float m = NEG_INF, l = 0.0f;
    f32x4 o[4] = {};
    for (int p = wave; p < t.parts; p += NW * UN) {
        float2 ml[UN];
        f32x4 y[UN][4];
#pragma unroll
        for (int k = 0; k < UN; ++k) {
            const float *at = from + min(p + k * NW, t.parts - 1) * stride;  // past the end: not added below
            ml[k] = *reinterpret_cast<const float2 *>(at + ROWS * D + lane * 2);
#pragma unroll
            for (int e = 0; e < 4; ++e) y[k][e] = *reinterpret_cast<const f32x4 *>(at + (b * 4 + e) * 256 + lane * 4);
        }
#pragma unroll
        for (int k = 0; k < UN; ++k) {
            if (p + k * NW >= t.parts) break;  // uniform
            const float top = fmaxf(m, ml[k].x), mu = top == NEG_INF ? 0.0f : top;
            const float f0 = exp2_(m - mu), f1 = exp2_(ml[k].x - mu);
            l = l * f0 + ml[k].y * f1;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = o[e] * f0 + y[k][e] * f1;
            m = top;
        }
    }
    mls[wave][lane] = float2{m, l};
#pragma unroll
    for (int e = 0; e < 4; ++e) os[wave][e][lane] = o[e];
    __syncthreads();
    float top = NEG_INF, z = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, mls[w][lane].x);
    const float mu = top == NEG_INF ? 0.0f : top;
    f32x4 sum = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const float f = exp2_(mls[w][lane].x - mu);
        z += mls[w][lane].y * f;
        sum += os[w][wave][lane] * f;
    }
    if (row >= rows) return;
    const int64_t token = t.token + (head0 + row) / G, head = kvhead * G + (head0 + row) % G;
    const float inv = z == 0.0f ? 0.0f : 1.0f / z;
    char *to = static_cast<char *>(a.out) + (token * a.out_stride + head * D + b * 32 + wave * 8 + h * 4) * 2;
    *reinterpret_cast<u32x2 *>(to) = u32x2{pack2<F16>(mean<F16>(sum[0] * inv), mean<F16>(sum[1] * inv)),
                                           pack2<F16>(mean<F16>(sum[2] * inv), mean<F16>(sum[3] * inv))};
    if (a.lse && wave == 0 && h == 0 && b == 0) a.lse[token * a.heads + head] = z == 0.0f ? NEG_INF : (top + log2_(z)) * LN2;
}

int64_t tiles_of(const KvDev &c, int heads)
{
    const int64_t G = heads / c.kvh, rows = WAVES * ROWS;
    return c.qs ? c.n_tokens * G / rows + c.n_seq : c.n_seq * ((G + rows - 1) / rows);
}

// A prefill's keys are split only where there are no more tiles than groups_of(dim), which bounds the
// workspace: groups + tiles slots a head, at most 2 groups.  With more, a long tile is one workgroup's: 64 sequences of 64
// new tokens, 32 heads on 8, one behind 32,768 keys and the others behind 1,024, take 632 us, with the
// same keys spread evenly 162.
// A tree's are split with any number of tiles: slots are numbered among the parts of split tiles, 4/3 groups at most, of 2/3
// groups tiles (find_part_tree).
// Neither's where a call has more than 512 sequences (PER_THREAD for each thread to look at) or a table of SHORT keys: 512 trees
// of 4 nodes behind 196 tokens, four of them behind 15,996, 32 heads on 8, 164 us, 513 of them 404.
Plan plan_of(const KvDev &c, int heads, int dim, int window, int nodes)
{
    Plan p = {(int)tiles_of(c, heads), 0, 1, 0, 0};
    // no tile has more parts than MIN_SPLIT goes into the keys that it can see
    int64_t keys = (int64_t)c.max_blocks * SAE_KV_BLOCK;
    if (window > 0) keys = std::min(keys, (int64_t)window + WAVES * ROWS + nodes + keys_of(dim));
    p.most = (int)std::min((keys + keys_of(dim)) / MIN_SPLIT, (int64_t)groups_of(dim));
    const bool few = (int64_t)p.tiles * c.kvh <= groups_of(dim);
    if ((few || nodes > 0) && c.n_seq <= PER_THREAD * WAVES * SAE_WAVE && keys > SHORT) {
        p.groups = std::max(groups_of(dim) / c.kvh, 1);
        p.slots = few ? p.groups + p.tiles : 2 * p.groups;
        p.joins = std::min(p.tiles, 2 * p.groups / 3 + 1);  // (each has two parts, of 3/4 of a share at least)
    }
    return p;
}

template <int TYPE, int D>
hipError_t launch_tree_join(const KvDev &c, const AttnArgs &a, const Plan &p, hipStream_t s)
{
    const int64_t rows = std::min((int64_t)a.max_nodes * (a.heads / c.kvh), (int64_t)WAVES * ROWS);  // of a tile at most
    hipLaunchKernelGGL((k_tree_join<TYPE, D>), dim3((unsigned)(p.joins * c.kvh), D / 32, (unsigned)((rows + ROWS - 1) / ROWS)),
                       dim3(4 * SAE_WAVE), 0, s, c, a, p);
    return hipGetLastError();
}

template <int TYPE, int D, bool TREE>
hipError_t launch(const KvDev &c, const AttnArgs &a, hipStream_t s)
{
    const Plan p = plan_of(c, a.heads, D, a.window, TREE ? a.max_nodes : 0);
    if (!p.groups) {
        hipLaunchKernelGGL((k_prefill<TYPE, D, WAVES, false, TREE>), dim3(p.tiles * c.kvh), dim3(WAVES * SAE_WAVE), 0, s, c, a, p);
        return hipGetLastError();
    }
    // parts: at most a share of the work each, rounded up for every tile
    const unsigned grid = (unsigned)((p.groups + p.tiles) * c.kvh);
    hipLaunchKernelGGL((k_prefill<TYPE, D, WAVES, true, TREE>), dim3(grid), dim3(WAVES * SAE_WAVE), 0, s, c, a, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if constexpr (TREE) return launch_tree_join<TYPE, D>(c, a, p, s);
    hipLaunchKernelGGL((k_prefill_join<TYPE, D, WAVES>), dim3(grid, D / 32), dim3(WAVES * SAE_WAVE), 0, s, c, a, p);
    return hipGetLastError();
}

template <int TYPE, bool TREE>
hipError_t launch_dim(const KvDev &c, const AttnArgs &a, int dim, hipStream_t s)
{
    return dim == 64 ? launch<TYPE, 64, TREE>(c, a, s) : dim == 128 ? launch<TYPE, 128, TREE>(c, a, s) : launch<TYPE, 256, TREE>(c, a, s);
}

}  // namespace
