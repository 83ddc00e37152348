// What the kernels that move new tokens' rows into and out of the paged cache share:
// the tiles of a call, places in a page, roundings.  A tile is one sequence's part of one
// page (up to 16 tokens).
#pragma once

#include "kv_cache.h"

namespace {

constexpr int THREADS = 256;

__device__ __forceinline__ float half_to_float(uint32_t h)
{
    _Float16 x;
    const uint16_t b = (uint16_t)h;
    __builtin_memcpy(&x, &b, 2);
    return (float)x;
}

// Rounds to f16, to its largest value where that is passed (NaN stays NaN).
__device__ __forceinline__ uint32_t float_to_half_sat(float x)
{
    const float y = x > 65504.0f ? 65504.0f : x < -65504.0f ? -65504.0f : x;
    const _Float16 h = (_Float16)y;
    uint16_t b;
    __builtin_memcpy(&b, &h, 2);
    return b;
}

// Rounds to bf16, nearest even (NaN stays NaN).
__device__ __forceinline__ uint32_t float_to_bf16(float x)
{
    const __bf16 h = (__bf16)x;
    uint16_t b;
    __builtin_memcpy(&b, &h, 2);
    return b;
}

template <int DT>
__device__ __forceinline__ float wide(uint32_t h)
{
    return DT == SAE_KV_BF16 ? __uint_as_float(h << 16) : half_to_float(h);
}

struct Place {
    int64_t block;  // pool block, -1: none
    int t_lo, t_hi; // tokens of the page that belong to the call: [t_lo, t_hi)
    int row0;       // row of token t is row0 + t (row0 may be negative)
    int pos0;       // position of token t is pos0 + t
    bool none;      // nothing to do
    // rows whose position would be negative: [dead0, dead1)
    int dead0, dead1;
};

// The sequence of a tile and what is known of it, found by the whole workgroup: its
// threads look at 256 sequences in one round trip.
struct Seq {
    int r, q0, q1, len, inst;  // r < 0: none (a q_start that decreases)
};

__device__ __forceinline__ Seq find_seq(const KvDev &c, int64_t tile)
{
    __shared__ Seq found;
    __shared__ int below[THREADS / SAE_WAVE];
    if (!c.qs) {
        const int r = (int)tile;
        return {r, r, r + 1, c.len[r], c.inst ? c.inst[r] : 0};
    }
    // tiles before sequence r: at least the pages that those touch
    auto before = [&](int r, int q) { return (int64_t)(q >> 4) + 2ll * r; };
    int lo = 0, n = c.n_seq;
    while (n > THREADS) {  // the answer lies in [lo, lo + n)
        const int step = (n + THREADS - 1) / THREADS, r = lo + (int)threadIdx.x * step;
        const uint64_t m = __ballot(r < lo + n && before(r, c.qs[r]) <= tile);
        if (__lane_id() == 0) below[threadIdx.x / SAE_WAVE] = __popcll((long long)m);
        __syncthreads();
        int count = 0;
#pragma unroll
        for (int w = 0; w < THREADS / SAE_WAVE; ++w) count += below[w];
        __syncthreads();
        const int end = lo + n;
        lo += max(count - 1, 0) * step;
        n = min(step, end - lo);
    }
    if (threadIdx.x == 0) found.r = -1;
    __syncthreads();
    const int r = lo + (int)threadIdx.x;
    if (r < lo + n) {
        const Seq s = {r, c.qs[r], c.qs[r + 1], c.len[r], c.inst ? c.inst[r] : 0};
        if (before(r, s.q0) <= tile && (r + 1 == c.n_seq || tile < before(r + 1, s.q1))) found = s;
    }
    __syncthreads();
    return {__builtin_amdgcn_readfirstlane(found.r), __builtin_amdgcn_readfirstlane(found.q0),
            __builtin_amdgcn_readfirstlane(found.q1), __builtin_amdgcn_readfirstlane(found.len),
            __builtin_amdgcn_readfirstlane(found.inst)};
}

// Tile -> sequence and page.
__device__ __forceinline__ Place place_of(const KvDev &c, int64_t tile)
{
    Place p = {};
    const Seq s = find_seq(c, tile);
    p.none = true;
    if (s.r < 0) return p;
    const int r = s.r;
    // the tile's number among its sequence's
    const int64_t sub = c.qs ? tile - ((int64_t)(s.q0 >> 4) + 2ll * r) : 0;
    const int first = min(max(s.q0, 0), c.n_tokens), count = min(max(s.q1, first), c.n_tokens) - first;
    const int len = kv::checked_len(c, s.len);
    const int start = len - count;  // position of the first new token; < 0: the first -start rows have no place
    const int pos0 = max(start, 0);
    p.none = sub < 0 || count == 0 || ((pos0 >> 4) + sub) * SAE_KV_BLOCK >= len;
    const int page = p.none ? 0 : (pos0 >> 4) + (int)sub;
    p.t_lo = max(pos0 - (page << 4), 0);
    p.t_hi = min(len - (page << 4), SAE_KV_BLOCK);
    p.row0 = first - start + (page << 4);
    p.pos0 = page << 4;
    p.block = -1;
    if (!p.none) p.block = kv::pool_block(c, kv::inst_base(c, s.inst), c.ids[(int64_t)r * c.max_blocks + page]);
    p.dead0 = p.dead1 = first;
    if (sub == 0 && start < 0) p.dead1 = first + min(count, -start);
    return p;
}

// Byte offset in a page of the value unit (4 tokens tg, dimension d).
template <int TYPE>
__device__ __forceinline__ int v_unit(int d, int tg)
{
    constexpr int E = TYPE == SAE_KV_FP8 ? 1 : 2, ND = TYPE == SAE_KV_FP8 ? 2 : 1;
    return (((d / (16 * ND) * 16 + d % 16) * 2 + (tg & 1)) * ND + d / 16 % ND) * 8 * E + (tg >> 1) * 4 * E;
}

// Maximum over the D / 8 lanes that hold one token's row.
template <int D>
__device__ __forceinline__ float row_max(float x)
{
#pragma unroll
    for (int o = 1; o < D / 8; o <<= 1) x = fmaxf(x, __shfl_xor(x, o));
    return x;
}

// The scale byte for the largest finite |x| of a row (see sae_kv_write).
__device__ __forceinline__ uint32_t scale_byte(float top)
{
    if (top == 0.0f) return 127;
    int e;
    const float m = frexpf(top, &e);  // top = m 2^e, m in [0.5, 1)
    return (uint32_t)(max(e - 9 + (m > 0.875f ? 1 : 0), -126) + 127);
}

// 8 values times `inv` as e4m3.
__device__ __forceinline__ u32x2 to_e4m3(const float (&f)[8], float inv)
{
    u32x2 r;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        int w = 0;
        w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j] * inv, f[4 * j + 1] * inv, w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j + 2] * inv, f[4 * j + 3] * inv, w, true);
        r[j] = (uint32_t)w;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (!(fabsf(f[j]) < __builtin_inff())) r[j / 4] |= 0x7Fu << (8 * (j & 3));  // NaN: 0x7F or 0xFF
    return r;
}

// 8 values of a row quantised; every lane of the row takes part.
template <int D, int DT>
__device__ __forceinline__ u32x2 quantise(u32x4 x, uint32_t &byte)
{
    float f[8], top = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        f[j] = wide<DT>((x[j / 2] >> (16 * (j & 1))) & 0xFFFFu);
        const float a = fabsf(f[j]);
        if (a < __builtin_inff()) top = fmaxf(top, a);  // false for infinities and NaN
    }
    byte = scale_byte(row_max<D>(top));
    return to_e4m3(f, __uint_as_float((254u - byte) << 23));  // 2^(127 - byte): byte is 1 .. 247
}

template <int DT>
__device__ __forceinline__ uint32_t narrow(float x)
{
    return DT == SAE_KV_BF16 ? float_to_bf16(x) : float_to_half_sat(x);
}

// Tiles of a call: an upper bound that needs no lengths.  A sequence of n new
// tokens touches at most (n + 14) / 16 + 1 <= n / 16 + 2 pages.
inline unsigned tiles_of(const KvDev &c) { return (unsigned)(c.qs ? (c.n_tokens >> 4) + 2ll * c.n_seq : c.n_seq); }

}  // namespace
