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
#include "kv_page.h"

namespace {

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

dim3 grid_of(const KvDev &c, int dim) { return dim3(tiles_of(c), (unsigned)((c.kvh * (dim / 2) + THREADS - 1) / THREADS)); }

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
