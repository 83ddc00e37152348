// Writing and reading the paged key-value cache.
//
// A call's new tokens are taken page by page: a tile is one sequence's part of
// one page (up to 16 tokens) of every head.  A thread owns 4 consecutive tokens
// (one token group of the value layout) x 8 dimensions: it moves 4 row pieces of
// 16 bytes each of keys and of values, so rows are read (or written) in runs of
// 2 head_dim bytes, and the value page's units of 4 tokens x 1 dimension are a
// 4 x 8 transposition in its own registers, with no LDS and no shuffles.
//
// Bound by memory: a token and head is read once and written once (counters agree:
// 94 MB written for 93 MB of cache, 334 MB for 334 MB of rows).  45,200 tokens of 8
// heads of 128 quantised to 8 bits: 71 us, 3.9 TB/s of rows read and cache written;
// read back: 66 us, 4.2 TB/s; 81,600 tokens read: 104 us, 4.8 TB/s, what a copy
// reaches; 45,200 tokens of a 16-bit cache: 92 us and 4.0 TB/s written, 76 and 4.9
// read.  Stores of 4 or 8 bytes (a value unit) touch each line several times, which L2
// merges; gathering whole pages in LDS first would not lower the bytes.  A decode step's
// write (256 tokens) is 5.4-6.8 us: launch and three dependent round trips (sequence,
// table entry, rows).
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
    const float inv = __uint_as_float((254u - byte) << 23);  // 2^(127 - byte): byte is 1 .. 247
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

template <int TYPE, int D, int DT>
__global__ void __launch_bounds__(THREADS)
k_kv_write(KvDev c, const uint16_t *k, int64_t k_stride, const uint16_t *v, int64_t v_stride)
{
    constexpr int NCH = D / 8, PER_HEAD = 4 * NCH;  // threads of a page: [token group][piece]
    constexpr int E = TYPE == SAE_KV_FP8 ? 1 : 2;
    const Place p = place_of(c, blockIdx.x);
    if (p.none || p.block < 0) return;  // the whole workgroup
    const int at = blockIdx.y * THREADS + threadIdx.x;
    const int head = at / PER_HEAD, tg = at / NCH % 4, ch = at % NCH;
    // a wave holds whole rows (NCH lanes): heads past the last one leave together
    if (head >= c.kvh) return;
    u32x4 xk[4], xv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = tg * 4 + i;
        xk[i] = xv[i] = u32x4{0, 0, 0, 0};
        if (t >= p.t_lo && t < p.t_hi) {
            const int64_t row = (int64_t)p.row0 + t;
            xk[i] = *reinterpret_cast<const u32x4 *>(k + row * k_stride + head * D + ch * 8);
            xv[i] = *reinterpret_cast<const u32x4 *>(v + row * v_stride + head * D + ch * 8);
        }
    }
    char *kp = c.k + p.block * c.block_bytes + (int64_t)head * (SAE_KV_BLOCK * D * E);
    char *vp = c.v + p.block * c.block_bytes + (int64_t)head * (SAE_KV_BLOCK * D * E);
    const bool whole = tg * 4 >= p.t_lo && tg * 4 + 4 <= p.t_hi;
    if constexpr (TYPE == SAE_KV_FP8) {
        uint32_t bk[4], bv[4];
        u32x2 qk[4], qv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            qk[i] = quantise<D, DT>(xk[i], bk[i]);
            qv[i] = quantise<D, DT>(xv[i], bv[i]);
        }
        const int64_t sc = p.block * c.scale_stride + head * SAE_KV_BLOCK;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = tg * 4 + i;
            if (t < p.t_lo || t >= p.t_hi) continue;
            *reinterpret_cast<u32x2 *>(kp + (ch / 2) * 256 + t * 16 + (ch & 1) * 8) = qk[i];
            if (ch == 0) {
                c.ks[sc + t] = (uint8_t)bk[i];
                c.vs[sc + t] = (uint8_t)bv[i];
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t u = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) u |= ((qv[i][j / 4] >> (8 * (j & 3))) & 0xFFu) << (8 * i);
            char *to = vp + v_unit<TYPE>(ch * 8 + j, tg);
            if (whole) *reinterpret_cast<uint32_t *>(to) = u;
            else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = tg * 4 + i;
                    if (t >= p.t_lo && t < p.t_hi) to[i] = (char)(u >> (8 * i));
                }
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = tg * 4 + i;
            if (t >= p.t_lo && t < p.t_hi) *reinterpret_cast<u32x4 *>(kp + ch * 256 + t * 16) = xk[i];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t h[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = (xv[i][j / 2] >> (16 * (j & 1))) & 0xFFFFu;
            uint16_t *to = reinterpret_cast<uint16_t *>(vp + v_unit<TYPE>(ch * 8 + j, tg));
            if (whole) *reinterpret_cast<u32x2 *>(to) = u32x2{h[0] | h[1] << 16, h[2] | h[3] << 16};
            else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = tg * 4 + i;
                    if (t >= p.t_lo && t < p.t_hi) to[i] = (uint16_t)h[i];
                }
            }
        }
    }
}

template <int DT>
__device__ __forceinline__ uint32_t narrow(float x)
{
    return DT == SAE_KV_BF16 ? float_to_bf16(x) : float_to_half_sat(x);
}

template <int TYPE, int D, int DT>
__global__ void __launch_bounds__(THREADS)
k_kv_read(KvDev c, uint16_t *k, int64_t k_stride, uint16_t *v, int64_t v_stride)
{
    constexpr int NCH = D / 8, PER_HEAD = 4 * NCH;
    constexpr int E = TYPE == SAE_KV_FP8 ? 1 : 2;
    const Place p = place_of(c, blockIdx.x);
    const int at = blockIdx.y * THREADS + threadIdx.x;
    const int head = at / PER_HEAD, tg = at / NCH % 4, ch = at % NCH;
    if (head >= c.kvh) return;
    const u32x4 zero = {0, 0, 0, 0};
    for (int row = p.dead0 + tg; row < p.dead1; row += 4) {  // rows without a place
        *reinterpret_cast<u32x4 *>(k + row * k_stride + head * D + ch * 8) = zero;
        *reinterpret_cast<u32x4 *>(v + row * v_stride + head * D + ch * 8) = zero;
    }
    if (p.none) return;
    u32x4 xk[4] = {zero, zero, zero, zero}, xv[4] = {zero, zero, zero, zero};
    if (p.block >= 0 && tg * 4 < p.t_hi && tg * 4 + 4 > p.t_lo) {
        const char *kp = c.k + p.block * c.block_bytes + (int64_t)head * (SAE_KV_BLOCK * D * E);
        const char *vp = c.v + p.block * c.block_bytes + (int64_t)head * (SAE_KV_BLOCK * D * E);
        if constexpr (TYPE == SAE_KV_FP8) {
            const int64_t sc = p.block * c.scale_stride + head * SAE_KV_BLOCK + tg * 4;
            const uint32_t bk = *reinterpret_cast<const uint32_t *>(c.ks + sc);
            const uint32_t bv = *reinterpret_cast<const uint32_t *>(c.vs + sc);
            u32x2 qk[4];
            uint32_t qv[8];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                qk[i] = *reinterpret_cast<const u32x2 *>(kp + (ch / 2) * 256 + (tg * 4 + i) * 16 + (ch & 1) * 8);
#pragma unroll
            for (int j = 0; j < 8; ++j) qv[j] = *reinterpret_cast<const uint32_t *>(vp + v_unit<TYPE>(ch * 8 + j, tg));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // a power of two: the products are exact in fp32
                const float sk = __uint_as_float(((bk >> (8 * i)) & 0xFFu) << 23);
                const float sv = __uint_as_float(((bv >> (8 * i)) & 0xFFu) << 23);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float fk = __builtin_amdgcn_cvt_f32_fp8((int)(qk[i][j / 4] >> (8 * (j & 3))), 0) * sk;
                    const float fv = __builtin_amdgcn_cvt_f32_fp8((int)(qv[j] >> (8 * i)), 0) * sv;
                    xk[i][j / 2] |= narrow<DT>(fk) << (16 * (j & 1));
                    xv[i][j / 2] |= narrow<DT>(fv) << (16 * (j & 1));
                }
            }
        } else {
            u32x2 u[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) xk[i] = *reinterpret_cast<const u32x4 *>(kp + ch * 256 + (tg * 4 + i) * 16);
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = *reinterpret_cast<const u32x2 *>(vp + v_unit<TYPE>(ch * 8 + j, tg));
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    xv[i][j / 2] |= ((u[j][i / 2] >> (16 * (i & 1))) & 0xFFFFu) << (16 * (j & 1));
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = tg * 4 + i;
        if (t < p.t_lo || t >= p.t_hi) continue;
        const int64_t row = (int64_t)p.row0 + t;
        *reinterpret_cast<u32x4 *>(k + row * k_stride + head * D + ch * 8) = xk[i];
        *reinterpret_cast<u32x4 *>(v + row * v_stride + head * D + ch * 8) = xv[i];
    }
}

// Tiles of a call: an upper bound that needs no lengths.  A sequence of n new
// tokens touches at most (n + 14) / 16 + 1 <= n / 16 + 2 pages.
dim3 grid_of(const KvDev &c, int dim)
{
    const long long tiles = c.qs ? (c.n_tokens >> 4) + 2ll * c.n_seq : c.n_seq;
    return dim3((unsigned)tiles, (unsigned)((c.kvh * (dim / 2) + THREADS - 1) / THREADS));
}

template <int TYPE, int D, int DT, bool WRITE>
void launch(const KvDev &c, void *k, int64_t ks, void *v, int64_t vs, hipStream_t s)
{
    if constexpr (WRITE)
        hipLaunchKernelGGL((k_kv_write<TYPE, D, DT>), grid_of(c, D), dim3(THREADS), 0, s, c, (const uint16_t *)k, ks,
                           (const uint16_t *)v, vs);
    else
        hipLaunchKernelGGL((k_kv_read<TYPE, D, DT>), grid_of(c, D), dim3(THREADS), 0, s, c, (uint16_t *)k, ks,
                           (uint16_t *)v, vs);
}

template <int D, bool WRITE>
void launch_types(const KvDev &c, int type, int dtype, void *k, int64_t ks, void *v, int64_t vs, hipStream_t s)
{
    // 16-bit values are moved as bits: one kernel for both types
    if (type != SAE_KV_FP8) launch<SAE_KV_BF16, D, SAE_KV_BF16, WRITE>(c, k, ks, v, vs, s);
    else if (dtype == SAE_KV_BF16) launch<SAE_KV_FP8, D, SAE_KV_BF16, WRITE>(c, k, ks, v, vs, s);
    else launch<SAE_KV_FP8, D, SAE_KV_F16, WRITE>(c, k, ks, v, vs, s);
}

template <bool WRITE>
hipError_t launch_dims(const KvDev &c, int type, int dim, int dtype, void *k, int64_t ks, void *v, int64_t vs,
                       hipStream_t s)
{
    if (dim == 64) launch_types<64, WRITE>(c, type, dtype, k, ks, v, vs, s);
    else if (dim == 128) launch_types<128, WRITE>(c, type, dtype, k, ks, v, vs, s);
    else launch_types<256, WRITE>(c, type, dtype, k, ks, v, vs, s);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_write(const KvDev &c, int type, int dim, int dtype, const void *k, int64_t k_stride,
                           const void *v, int64_t v_stride, hipStream_t s)
{
    return launch_dims<true>(c, type, dim, dtype, const_cast<void *>(k), k_stride, const_cast<void *>(v), v_stride, s);
}

hipError_t launch_kv_read(const KvDev &c, int type, int dim, int dtype, void *k, int64_t k_stride, void *v,
                          int64_t v_stride, hipStream_t s)
{
    return launch_dims<false>(c, type, dim, dtype, k, k_stride, v, v_stride, s);
}
