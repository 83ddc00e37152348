// New tokens' keys and values to their places in the paged cache, keys and queries turned by
// their positions' angles on the way.
//
//   pair i of a head's first R dimensions, (x, y) at (i, i + R / 2) or (2 i, 2 i + 1), becomes
//   f (x cos a - y sin a, x sin a + y cos a),  a = position * inv_freq[i]
//
// in fp32, rounded once: to the rows' type, or to the 8-bit cache's (a power-of-two scale from the
// turned row's largest value).  The angle is reduced in 64 bits: at position 10^6 a 32-bit product
// is off by 0.06 and more.
//
// A workgroup takes a part of a tile (one sequence's tokens of one page): it computes the cosines and sines
// of the tile's tokens once into LDS, for all of its heads, then each thread takes 4 tokens x
// two 16-byte pieces, the two that hold the pairs' halves, of keys and values or of queries.
//
// Bound by memory: 22,600 tokens of 32 and 8 heads of 128 into an 8-bit cache, 124 us: 509 MB (272
// fetched, 227 written, by the counters), 4.1 TB/s, where a copy reaches 5.1.  At 128 registers,
// four waves a SIMD (180, two waves: 141 us; the next rows or the first ones loaded ahead of the angles:
// spilled, 145 and more; 2, 3 or 5 items a thread: 121 to 127).  A step of 256 tokens is 8.2 us, one token 5.9: dependent round
// trips (sequence, table entry, positions, rows).
#include "kv_page.h"

namespace {

struct Append {
    const uint16_t *q, *k, *v;
    uint16_t *q_out;
    int64_t q_stride, out_stride, k_stride, v_stride;
    const int32_t *pos;
    const float *freq;
    float factor;
    int32_t turned, interleaved, heads;
};

// Cosine and sine of 2 pi `turns` times the factor, by their Taylor series on +-1/8 of a turn (next terms: 2e-9).
__device__ __forceinline__ float2 circle(double turns, float factor)
{
    turns -= __builtin_rint(turns);
    const double quarter = __builtin_rint(turns * 4.0);
    const float a = (float)((turns - quarter * 0.25) * 6.283185307179586476925), z = a * a;
    float s = __builtin_fmaf(z, 1.0f / 362880, -1.0f / 5040);
    s = __builtin_fmaf(z, s, 1.0f / 120);
    s = __builtin_fmaf(z, s, -1.0f / 6);
    s = __builtin_fmaf(z * a, s, a);
    float c = __builtin_fmaf(z, -1.0f / 3628800, 1.0f / 40320);
    c = __builtin_fmaf(z, c, -1.0f / 720);
    c = __builtin_fmaf(z, c, 1.0f / 24);
    c = __builtin_fmaf(z, c, -0.5f);
    c = __builtin_fmaf(z, c, 1.0f);
    const int n = (int)quarter & 3;
    const float x = n & 1 ? s : c, y = n & 1 ? c : s;
    return float2{(n == 1 || n == 2 ? -x : x) * factor, (n >= 2 ? -y : y) * factor};
}

template <int DT>
__device__ __forceinline__ void widen(u32x4 x, float (&f)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = wide<DT>((x[j / 2] >> (16 * (j & 1))) & 0xFFFFu);
}

// 8 values rounded to the rows' type (past f16's range: infinity).
template <int DT>
__device__ __forceinline__ u32x4 round8(const float (&f)[8])
{
    u32x4 x;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t w[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if constexpr (DT == SAE_KV_BF16) w[e] = float_to_bf16(f[2 * j + e]);
            else {
                const _Float16 h = (_Float16)f[2 * j + e];
                uint16_t b;
                __builtin_memcpy(&b, &h, 2);
                w[e] = b;
            }
        }
        x[j] = w[0] | w[1] << 16;
    }
    return x;
}

// The two pieces a, b of a token turned; cs: the token's cosines and sines, at: the first pair's number.
__device__ __forceinline__ void turn(float (&a)[8], float (&b)[8], const float2 *cs, int at, bool interleaved)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 t = cs[at + j];
        // interleaved: pairs 0..3 are in a, 4..7 in b
        float &x = interleaved ? (j < 4 ? a[2 * j] : b[2 * j - 8]) : a[j];
        float &y = interleaved ? (j < 4 ? a[2 * j + 1] : b[2 * j - 7]) : b[j];
        const float u = __builtin_fmaf(x, t.x, -(y * t.y)), w = __builtin_fmaf(x, t.y, y * t.x);
        x = u;
        y = w;
    }
}

// A token's row over LANES lanes quantised, 2 pieces a lane; returns the scale byte.
template <int LANES>
__device__ __forceinline__ uint32_t quantise2(const float (&a)[8], const float (&b)[8], u32x2 &qa, u32x2 &qb)
{
    float top = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float x = fabsf(a[j]), y = fabsf(b[j]);
        if (x < __builtin_inff()) top = fmaxf(top, x);  // false for infinities and NaN
        if (y < __builtin_inff()) top = fmaxf(top, y);
    }
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    const uint32_t byte = scale_byte(top);
    const float inv = __uint_as_float((254u - byte) << 23);
    qa = to_e4m3(a, inv);
    qb = to_e4m3(b, inv);
    return byte;
}

// A token's turned keys, 2 pieces, into the page.
template <int TYPE, int D, int DT>
__device__ __forceinline__ void put_key(const KvDev &c, const Place &p, int head, int t, int lane, const int (&ch)[2], bool turned,
                                        const u32x4 (&raw)[2], const float (&x)[8], const float (&y)[8])
{
    constexpr int E = TYPE == SAE_KV_FP8 ? 1 : 2;
    char *page = c.k + p.block * c.block_bytes + (int64_t)head * (SAE_KV_BLOCK * D * E);
    const bool there = t >= p.t_lo && t < p.t_hi;
    if constexpr (TYPE == SAE_KV_FP8) {
        u32x2 a, b;
        const uint32_t byte = quantise2<D / 16>(x, y, a, b);
        if (!there) return;
        *reinterpret_cast<u32x2 *>(page + (ch[0] / 2) * 256 + t * 16 + (ch[0] & 1) * 8) = a;
        *reinterpret_cast<u32x2 *>(page + (ch[1] / 2) * 256 + t * 16 + (ch[1] & 1) * 8) = b;
        if (lane == 0) c.ks[p.block * c.scale_stride + head * SAE_KV_BLOCK + t] = (uint8_t)byte;
    } else {
        if (!there) return;
        *reinterpret_cast<u32x4 *>(page + ch[0] * 256 + t * 16) = turned ? round8<DT>(x) : raw[0];
        *reinterpret_cast<u32x4 *>(page + ch[1] * 256 + t * 16) = turned ? round8<DT>(y) : raw[1];
    }
}

// Values of 4 tokens, 2 pieces each, into the page.
template <int TYPE, int D, int DT>
__device__ __forceinline__ void put_values(const KvDev &c, const Place &p, int head, int tg, int lane, const int (&ch)[2],
                                           const u32x4 (&raw)[4][2])
{
    constexpr int E = TYPE == SAE_KV_FP8 ? 1 : 2;
    char *page = c.v + p.block * c.block_bytes + (int64_t)head * (SAE_KV_BLOCK * D * E);
    const bool whole = tg * 4 >= p.t_lo && tg * 4 + 4 <= p.t_hi;
    if constexpr (TYPE == SAE_KV_FP8) {
        u32x2 q[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = tg * 4 + i;
            float x[8], y[8];
            widen<DT>(raw[i][0], x);
            widen<DT>(raw[i][1], y);
            const uint32_t byte = quantise2<D / 16>(x, y, q[i][0], q[i][1]);
            if (lane == 0 && t >= p.t_lo && t < p.t_hi) c.vs[p.block * c.scale_stride + head * SAE_KV_BLOCK + t] = (uint8_t)byte;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                char *to = page + v_unit<TYPE>(ch[u] * 8 + j, tg);
                uint32_t y = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) y |= ((q[i][u][j / 4] >> (8 * (j & 3))) & 0xFFu) << (8 * i);
                if (whole) *reinterpret_cast<uint32_t *>(to) = y;
                else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (tg * 4 + i >= p.t_lo && tg * 4 + i < p.t_hi) to[i] = (char)(y >> (8 * i));
                }
            }
    } else {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                char *to = page + v_unit<TYPE>(ch[u] * 8 + j, tg);
                uint32_t h[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) h[i] = (raw[i][u][j / 2] >> (16 * (j & 1))) & 0xFFFFu;
                if (whole) *reinterpret_cast<u32x2 *>(to) = u32x2{h[0] | h[1] << 16, h[2] | h[3] << 16};
                else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (tg * 4 + i >= p.t_lo && tg * 4 + i < p.t_hi) reinterpret_cast<uint16_t *>(to)[i] = (uint16_t)h[i];
                }
            }
    }
}

template <int TYPE, int D, int DT>
__global__ void __launch_bounds__(THREADS, 4) k_kv_append(KvDev c, Append a)
{
    constexpr int LANES = D / 16;  // of a token's row
    __shared__ float2 cs[SAE_KV_BLOCK][D / 2];
    const Place p = place_of(c, blockIdx.x);
    const int start = blockIdx.y * THREADS + threadIdx.x, step = gridDim.y * THREADS;
    if (a.q_out)  // rows without a place
        for (int row = p.dead0; row < p.dead1; ++row)
            for (int i = start; i < a.heads * (D / 8); i += step)
                *reinterpret_cast<u32x4 *>(a.q_out + row * a.out_stride + i * 8) = u32x4{0, 0, 0, 0};
    if (p.none) return;
    // items: [key-value heads, then query heads][token groups of the tile][lanes of a row]
    const int tg0 = p.t_lo / 4, groups = (p.t_hi + 3) / 4 - tg0;
    const int kv_items = c.kvh * groups * LANES, items = kv_items + a.heads * groups * LANES;
    if ((int)blockIdx.y * THREADS >= items) return;
    const int half = a.turned / 2;
    for (int i = p.t_lo * half + threadIdx.x; i < p.t_hi * half; i += THREADS) {
        const int t = (int)((uint32_t)i / (uint32_t)half), j = i - t * half;
        const int pos = a.pos ? a.pos[p.row0 + t] : p.pos0 + t;
        cs[t][j] = circle((double)pos * ((double)a.freq[j] * 0.159154943091895335769), a.factor);
    }
    __syncthreads();
#pragma unroll 1
    for (int at = start; at < items; at += step) {
        const bool query = at >= kv_items;
        const int n = query ? at - kv_items : at, lane = n % LANES, g = n / LANES;
        const int head = (int)((uint32_t)g / (uint32_t)groups), tg = tg0 + g - head * groups;
        // the lane's two pieces
        const int h8 = half / 8;
        const bool turned = lane < h8, apart = turned && !a.interleaved;
        const int ch[2] = {apart ? lane : 2 * lane, apart ? lane + h8 : 2 * lane + 1};
        if (!query && p.block < 0) continue;
        auto load = [&](u32x4 (&x)[4][2], const uint16_t *from, int64_t stride) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = tg * 4 + i;
                const uint16_t *row = from + ((int64_t)p.row0 + t) * stride + head * D;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    x[i][u] = u32x4{0, 0, 0, 0};
                    if (t >= p.t_lo && t < p.t_hi) x[i][u] = *reinterpret_cast<const u32x4 *>(row + ch[u] * 8);
                }
            }
        };
        auto turn_token = [&](const u32x4 (&raw)[2], int t, float (&x)[8], float (&y)[8]) __attribute__((always_inline)) {
            widen<DT>(raw[0], x);
            widen<DT>(raw[1], y);
            if (turned && t >= p.t_lo && t < p.t_hi) {
                if (a.interleaved) turn(x, y, cs[t], lane * 8, true);
                else turn(x, y, cs[t], lane * 8, false);
            }
        };
        if (query) {
            u32x4 raw[4][2];
            load(raw, a.q, a.q_stride);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = tg * 4 + i;
                float x[8], y[8];
                turn_token(raw[i], t, x, y);
                if (t < p.t_lo || t >= p.t_hi) continue;
                uint16_t *to = a.q_out + ((int64_t)p.row0 + t) * a.out_stride + head * D;
                *reinterpret_cast<u32x4 *>(to + ch[0] * 8) = turned ? round8<DT>(x) : raw[i][0];
                *reinterpret_cast<u32x4 *>(to + ch[1] * 8) = turned ? round8<DT>(y) : raw[i][1];
            }
            continue;
        }
        u32x4 rk[4][2], rv[4][2];
        load(rk, a.k, a.k_stride);
        load(rv, a.v, a.v_stride);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[8], y[8];
            turn_token(rk[i], tg * 4 + i, x, y);
            put_key<TYPE, D, DT>(c, p, head, tg * 4 + i, lane, ch, turned, rk[i], x, y);
        }
        put_values<TYPE, D, DT>(c, p, head, tg, lane, ch, rv);
    }
}

template <int TYPE, int D, int DT>
hipError_t launch(const KvDev &c, const Append &a, hipStream_t s)
{
    // threads of a tile whose sequence has the batch's mean of new tokens
    const int64_t mean = c.qs ? (c.n_tokens + c.n_seq - 1) / c.n_seq : 1;
    const int64_t items = (int64_t)(c.kvh + a.heads) * (mean >= 16 ? 4 : (mean + 3) / 4) * (D / 16);
    hipLaunchKernelGGL((k_kv_append<TYPE, D, DT>), dim3(tiles_of(c), (unsigned)((items + THREADS - 1) / THREADS)),
                       dim3(THREADS), 0, s, c, a);
    return hipGetLastError();
}

template <int TYPE, int DT>
hipError_t launch_dim(const KvDev &c, const Append &a, int dim, hipStream_t s)
{
    return dim == 64 ? launch<TYPE, 64, DT>(c, a, s) : dim == 128 ? launch<TYPE, 128, DT>(c, a, s) : launch<TYPE, 256, DT>(c, a, s);
}

}  // namespace

hipError_t launch_kv_append(const KvDev &c, int type, int dim, int dtype, const AppendArgs &x, hipStream_t s)
{
    const Append a = {static_cast<const uint16_t *>(x.q), static_cast<const uint16_t *>(x.k), static_cast<const uint16_t *>(x.v),
                      static_cast<uint16_t *>(x.q_out), x.q_stride, x.out_stride, x.k_stride, x.v_stride, x.pos,
                      x.rope->inv_freq, x.rope->factor, x.rope->turned, x.rope->interleaved, x.heads};
    if (type == SAE_KV_BF16) return launch_dim<SAE_KV_BF16, SAE_KV_BF16>(c, a, dim, s);
    if (type == SAE_KV_F16) return launch_dim<SAE_KV_F16, SAE_KV_F16>(c, a, dim, s);
    return dtype == SAE_KV_BF16 ? launch_dim<SAE_KV_FP8, SAE_KV_BF16>(c, a, dim, s) : launch_dim<SAE_KV_FP8, SAE_KV_F16>(c, a, dim, s);
}
