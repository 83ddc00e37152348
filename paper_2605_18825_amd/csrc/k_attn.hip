// Attention of new tokens over the paged key-value cache.
//
// One wave per (new token, query head).  64 keys at a time: lane l takes key l's
// score (its products summed in fp32), the wave keeps the running maximum m and
// sum of a softmax, and lane l accumulates dimensions l, l + 64, ... of the output.
#include "kv_cache.h"

namespace {

template <int TYPE>
__device__ __forceinline__ float value_at(const char *p, int i)
{
    if constexpr (TYPE == SAE_KV_FP8) return __builtin_amdgcn_cvt_f32_fp8((int)reinterpret_cast<const uint8_t *>(p)[i], 0);
    else if constexpr (TYPE == SAE_KV_BF16) return (float)reinterpret_cast<const __bf16 *>(p)[i];
    else return (float)reinterpret_cast<const _Float16 *>(p)[i];
}

template <int TYPE, int D>
__global__ void __launch_bounds__(SAE_WAVE) k_attn_rows(KvDev c, AttnArgs a)
{
    constexpr int QT = TYPE == SAE_KV_FP8 ? SAE_KV_BF16 : TYPE;
    constexpr int E = TYPE == SAE_KV_FP8 ? 1 : 2, C = 16 / E;
    __shared__ float q[D], p[SAE_WAVE];
    __shared__ int64_t blk[SAE_WAVE / SAE_KV_BLOCK];
    const int row = blockIdx.x, head = blockIdx.y, lane = threadIdx.x;
    const int kvhead = head / (a.heads / c.kvh);
    const int r = c.qs ? kv::find_seq(c, row, 0, 0) : row;
    int first, count;
    kv::seq_rows(c, r, first, count);
    const int pos = kv::seq_len(c, r) - count + (row - first);  // of this query; may be negative
    const int lo = a.window > 0 ? max(0, pos - a.window + 1) : 0;
    const int64_t base = kv::seq_base(c, r);
    const char *qr = reinterpret_cast<const char *>(a.q) + (row * a.q_stride + head * D) * 2;
    for (int d = lane; d < D; d += SAE_WAVE) q[d] = value_at<QT>(qr, d);
    float m = -__builtin_inff(), sum = 0.0f, acc[D / SAE_WAVE] = {};
    for (int t0 = lo & ~(SAE_WAVE - 1); t0 <= pos; t0 += SAE_WAVE) {
        const int pg = t0 / SAE_KV_BLOCK + lane;
        if (lane < SAE_WAVE / SAE_KV_BLOCK)
            blk[lane] = pg * SAE_KV_BLOCK <= pos ? kv::pool_block(c, base, c.ids[(int64_t)r * c.max_blocks + pg]) : -1;
        __syncthreads();
        const int t = t0 + lane, tt = lane % SAE_KV_BLOCK;
        const int64_t b = blk[lane / SAE_KV_BLOCK];
        float s = -__builtin_inff();
        if (b >= 0 && t >= lo && t <= pos) {
            const char *kp = c.k + b * c.block_bytes + (int64_t)kvhead * (SAE_KV_BLOCK * D * E);
            float x = 0.0f;
            for (int d = 0; d < D; ++d) x += q[d] * value_at<TYPE>(kp, (d / C * SAE_KV_BLOCK + tt) * C + d % C);
            if (TYPE == SAE_KV_FP8)
                x *= __uint_as_float((uint32_t)c.ks[b * c.scale_stride + kvhead * SAE_KV_BLOCK + tt] << 23);
            s = x * a.scale;
        }
        float top = s;
        for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
        const float mn = fmaxf(m, top);
        const float mu = mn == -__builtin_inff() ? 0.0f : mn;  // nothing seen yet
        const float w = __expf(s - mu), old = __expf(m - mu);
        float ws = w;
        for (int o = 32; o; o >>= 1) ws += __shfl_xor(ws, o);
        sum = sum * old + ws;
        m = mn;
        float pv = w;
        if (TYPE == SAE_KV_FP8 && w != 0.0f)
            pv *= __uint_as_float((uint32_t)c.vs[b * c.scale_stride + kvhead * SAE_KV_BLOCK + tt] << 23);
        p[lane] = pv;
        __syncthreads();
        for (int i = 0; i < D / SAE_WAVE; ++i) acc[i] *= old;
        for (int j = 0; j < SAE_WAVE; ++j) {
            const float pj = p[j];
            if (blk[j / SAE_KV_BLOCK] < 0 || t0 + j < lo || t0 + j > pos) continue;  // uniform; its value may be NaN
            const char *vp = c.v + blk[j / SAE_KV_BLOCK] * c.block_bytes + (int64_t)kvhead * (SAE_KV_BLOCK * D * E);
            const int jt = j % SAE_KV_BLOCK;
            for (int i = 0; i < D / SAE_WAVE; ++i) {
                const int d = lane + SAE_WAVE * i;
                const int at = (((d / (2 * C) * 16 + d % 16) * 2 + jt / 4 % 2) * (C / 8) + d / 16 % (C / 8)) * 8 +
                               jt / 8 * 4 + jt % 4;
                acc[i] += pj * value_at<TYPE>(vp, at);
            }
        }
        __syncthreads();
    }
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    for (int i = 0; i < D / SAE_WAVE; ++i) {
        const float o = acc[i] * inv;
        const int64_t at = row * a.out_stride + head * D + lane + SAE_WAVE * i;
        if (QT == SAE_KV_BF16) reinterpret_cast<__bf16 *>(a.out)[at] = (__bf16)o;
        else reinterpret_cast<_Float16 *>(a.out)[at] = (_Float16)o;
    }
    if (a.lse && lane == 0)
        a.lse[(int64_t)row * a.heads + head] = sum == 0.0f ? -__builtin_inff() : m + __logf(sum);
}

template <int TYPE>
void launch_dim(const KvDev &c, const AttnArgs &a, int dim, hipStream_t s)
{
    const dim3 grid(c.n_tokens, a.heads);
    if (dim == 64) hipLaunchKernelGGL((k_attn_rows<TYPE, 64>), grid, dim3(SAE_WAVE), 0, s, c, a);
    else if (dim == 128) hipLaunchKernelGGL((k_attn_rows<TYPE, 128>), grid, dim3(SAE_WAVE), 0, s, c, a);
    else hipLaunchKernelGGL((k_attn_rows<TYPE, 256>), grid, dim3(SAE_WAVE), 0, s, c, a);
}

}  // namespace

size_t attn_work_bytes(int, int heads, int kvh, int dim) { return decode_work_bytes(heads, kvh, dim); }

hipError_t launch_attn(const KvDev &c, const AttnArgs &a, int type, int dim, bool decode, hipStream_t s)
{
    if (decode) return launch_decode(c, a, type, dim, s);
    if (type == SAE_KV_BF16) launch_dim<SAE_KV_BF16>(c, a, dim, s);
    else if (type == SAE_KV_F16) launch_dim<SAE_KV_F16>(c, a, dim, s);
    else launch_dim<SAE_KV_FP8>(c, a, dim, s);
    return hipGetLastError();
}
