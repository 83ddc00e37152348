// The paged key-value cache as the kernels see it: layout, tables and the
// lookups shared by k_kv.hip, k_decode.hip and k_prefill.hip.
#pragma once

#include "sae_internal.h"

// A sae_kv and a sae_seqs, checked, strides resolved to bytes.
struct KvDev {
    char *k, *v;
    uint8_t *ks, *vs;
    int64_t block_bytes;   // from a block's pages to the next block's, in k and in v
    int64_t scale_stride;
    const int32_t *ids, *inst, *len, *qs;
    uint32_t *status;
    int32_t n_inst, bpi, kvh, n_seq, max_blocks, n_tokens;
};

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

namespace kv {

__device__ __forceinline__ void report(const KvDev &c)
{
    if (c.status) atomicOr(c.status, (uint32_t)SAE_ST_BAD_BLOCK);
}

// A sequence's length; one that its table cannot hold is reported and cut.
__device__ __forceinline__ int checked_len(const KvDev &c, int n)
{
    const long long most = (long long)c.max_blocks * SAE_KV_BLOCK;
    if (n < 0 || n > most) {
        report(c);
        return n < 0 ? 0 : (int)most;
    }
    return n;
}

__device__ __forceinline__ int seq_len(const KvDev &c, int r) { return checked_len(c, c.len[r]); }

// First pool block of instance i, or -1.
__device__ __forceinline__ int64_t inst_base(const KvDev &c, int i)
{
    if (i < 0 || i >= c.n_inst) {
        report(c);
        return -1;
    }
    return (int64_t)i * c.bpi;
}

// First pool block of sequence r's instance, or -1.
__device__ __forceinline__ int64_t seq_base(const KvDev &c, int r) { return inst_base(c, c.inst ? c.inst[r] : 0); }

// Pool block for table entry `id` of a sequence with that base; -1 for none.
__device__ __forceinline__ int64_t pool_block(const KvDev &c, int64_t base, int id)
{
    if (id >= c.bpi) report(c);
    return base < 0 || id < 0 || id >= c.bpi ? -1 : base + id;
}

// Rows of sequence r in the call's arrays: [first, first + count), inside
// 0 .. n_tokens whatever q_start holds.
__device__ __forceinline__ void seq_rows(const KvDev &c, int r, int &first, int &count)
{
    if (!c.qs) {
        first = r;
        count = 1;
        return;
    }
    const int a = min(max(c.qs[r], 0), c.n_tokens), b = min(max(c.qs[r + 1], a), c.n_tokens);
    first = a;
    count = b - a;
}

}  // namespace kv

hipError_t launch_kv_write(const KvDev &c, int type, int dim, int dtype, const void *k, int64_t k_stride,
                           const void *v, int64_t v_stride, hipStream_t s);
hipError_t launch_kv_read(const KvDev &c, int type, int dim, int dtype, void *k, int64_t k_stride, void *v,
                          int64_t v_stride, hipStream_t s);

// An append, checked.  Strides in values; q and q_out may be null together.
struct AppendArgs {
    const sae_rope *rope;
    const int32_t *pos;
    int32_t heads;
    const void *q, *k, *v;
    void *q_out;
    int64_t q_stride, out_stride, k_stride, v_stride;
};
hipError_t launch_kv_append(const KvDev &c, int type, int dim, int dtype, const AppendArgs &x, hipStream_t s);

// One attention call, checked.  Strides in values.
struct AttnArgs {
    const void *q;
    void *out;
    float *lse;
    int64_t q_stride, out_stride;
    float scale;
    int32_t window, heads;
    void *work;
    // sae_attn_tree only
    const int32_t *parent;
    int32_t max_nodes;
};
hipError_t launch_decode(const KvDev &c, const AttnArgs &a, int type, int dim, hipStream_t s);
hipError_t launch_tree(const KvDev &c, const AttnArgs &a, int type, int dim, hipStream_t s);
hipError_t launch_prefill(const KvDev &c, const AttnArgs &a, int type, int dim, hipStream_t s);
// A sampling call, checked.
struct SampleArgs {
    const void *logits;
    int64_t stride;
    sae_sampling settings;
    const float *u;
    int32_t *token, *kept;
    float *prob;
    void *work;
};
hipError_t launch_sample(int rows, int vocab, int dtype, const SampleArgs &x, hipStream_t s);
size_t sample_work_bytes(int rows, int vocab);

size_t decode_work_bytes(int heads, int kvh, int dim);
size_t prefill_work_bytes(int kvh, int dim);
bool prefill_fits(const KvDev &c, int heads);
