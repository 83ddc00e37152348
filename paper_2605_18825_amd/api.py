"""Python binding of libsae with the C ABI's names.

Argument marshalling only: every operation runs in the HIP library.  Device
buffers are torch tensors on the current HIP device; the stream is torch's
current stream unless one is passed.
"""
import ctypes

import torch

from . import _lib
from ._lib import IVL_CAP, N_BINS, SaeConfig, SaeCounters, SaeError, SaeKv, SaeParams, SaePool, SaePredictor, SaeRope, SaeSampling, SaeSeqs  # noqa: F401

KIND_EVICT_FIRST, KIND_STRUCTURAL, KIND_LOGNORMAL, KIND_RECENCY = 0, 1, 2, 3
META_VALID, META_LEAF, META_REF = 0x40, 0x80, 0x100
PM_TOUCH, PM_STATS, PM_INTERVALS = 1, 2, 4
SS_COMMIT, SS_ENGINE_SCAN, SS_ENGINE_BATCHED, SS_FORCE_FALLBACK, SS_CASCADE = 1, 2, 4, 8, 16
FB_FORCE = 1
HINT_DECODE, HINT_UNTEMPLATED, HINT_MULTI_TURN, HINT_AGENTIC, HINT_CONVERSATION, HINT_SHARED_PREFIX = 1, 2, 4, 8, 16, 32
ROLE_EVICT, ROLE_STRUCT, ROLE_CHAT, ROLE_AGENT = 0, 1, 2, 3
LEARN_TOKEN_WEIGHTS, LEARN_QUEUE_WEIGHTS, LEARN_LOGNORMAL, LEARN_DECAY_POWER = 1, 2, 4, 8
LEARN_TOKEN_EMA, LEARN_QUEUE_REL = 16, 32
# the paper's initial token weights (system, user, tool, response, cot), Sec. 5
PAPER_INIT_W = (2.0, 1.5, 1.0, 1.0, 0.1)
ST_NAMES = {1: "INDEX_FULL", 2: "GHOST_FULL", 4: "BAD_OFFSET", 8: "FUTURE_ACCESS",
            16: "SLOT_BUSY", 32: "SELECT_FALLBACK", 64: "BAD_BLOCK", 128: "BAD_HASH", 256: "BAD_TREE"}


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise SaeError("expected a device tensor")
    if not t.is_contiguous():
        raise SaeError("expected a contiguous tensor")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _check(ctx, st):
    if st != 0:
        L = _lib.load()
        msg = L.sae_last_error(ctx).decode()
        raise SaeError("%s: %s" % (L.sae_status_str(st).decode(), msg))


# --------------------------------------------------------------------- layout
def pack_meta(queue, tau, ntok, valid=True, leaf=True, ref=False):
    """uint16 meta (as int32 tensor values): queue | tau<<3 | flags | (ntok-1)<<9."""
    m = (queue.to(torch.int32) & 7) | ((tau.to(torch.int32) & 7) << 3) | (((ntok.to(torch.int32) - 1) & 15) << 9)

    def flag(v, bit):
        if isinstance(v, torch.Tensor):
            return v.to(torch.int32) * bit
        return bit if v else 0
    return m | flag(valid, META_VALID) | flag(leaf, META_LEAF) | flag(ref, META_REF)


def meta_to_u16(m):
    """int32 values in [0, 65535] -> int16 tensor holding the same bits."""
    return (m.to(torch.int32) & 0xFFFF).to(torch.int16)


def unpack_meta(meta16):
    m = meta16.to(torch.int32) & 0xFFFF
    return dict(queue=m & 7, tau=(m >> 3) & 7, valid=(m & META_VALID) != 0, leaf=(m & META_LEAF) != 0,
                ref=(m & META_REF) != 0, ntok=((m >> 9) & 15) + 1)


def pack_off(ob, omax):
    return ((omax.to(torch.int64) << 16) | (ob.to(torch.int64) & 0xFFFF)).to(torch.int64)


def off_to_u32(off):
    """int64 values in [0, 2^32) -> int32 tensor holding the same bits."""
    return (off - ((off >= 2 ** 31).to(torch.int64) << 32)).to(torch.int32)


# ----------------------------------------------------------------- the C ABI
def sae_create(n_instances, blocks_per_instance, queue_kinds, max_k, ghost_window=0, index_log2=0, max_requests=0):
    L = _lib.load()
    cfg = SaeConfig()
    cfg.n_instances = n_instances
    cfg.blocks_per_instance = blocks_per_instance
    cfg.n_queues = len(queue_kinds)
    for i, k in enumerate(queue_kinds):
        cfg.queue_kind[i] = int(k)
    cfg.max_k = max_k
    cfg.ghost_window = ghost_window
    cfg.index_log2 = index_log2
    cfg.max_requests = max_requests
    out = ctypes.c_void_p()
    st = L.sae_create(ctypes.byref(cfg), ctypes.byref(out))
    if st != 0:
        raise SaeError("sae_create: %s: %s" % (L.sae_status_str(st).decode(), L.sae_last_error(None).decode()))
    return out


def sae_destroy(ctx):
    _check(ctx, _lib.load().sae_destroy(ctx))


def sae_bind_pool(ctx, last_access, meta, off, hash, parent, child_count, ref_count, access_count):
    p = SaePool()
    for name, t in (("last_access", last_access), ("meta", meta), ("off", off), ("hash", hash),
                    ("parent", parent), ("child_count", child_count), ("ref_count", ref_count),
                    ("access_count", access_count)):
        setattr(p, name, _ptr(t).value)
    _check(ctx, _lib.load().sae_bind_pool(ctx, ctypes.byref(p)))


def make_params(n_queues, w=1.0, alpha=1.0, mu=0.0, sigma=1.0, gamma=1.0, eta=0.01, temperature=1.0,
                beta=0.1, K=32, learn=LEARN_TOKEN_WEIGHTS | LEARN_QUEUE_WEIGHTS, beta_ln=0.1):
    p = SaeParams()

    def fill(arr, v, n):
        vals = list(v) if hasattr(v, "__len__") else [v] * n
        for i in range(len(arr)):
            arr[i] = float(vals[i]) if i < len(vals) else (1.0 if arr is p.sigma else 0.0)
    fill(p.w, w, 5)
    fill(p.alpha, alpha, n_queues)
    fill(p.mu, mu, n_queues)
    fill(p.sigma, sigma, n_queues)
    for i in range(n_queues, 8):
        p.alpha[i] = 1.0
        p.sigma[i] = 1.0
    p.gamma, p.eta, p.temperature, p.beta, p.beta_ln = gamma, eta, temperature, beta, beta_ln
    p.K, p.learn = int(K), int(learn)
    return p


def sae_set_params(ctx, inst, params, stream=None):
    _check(ctx, _lib.load().sae_set_params(ctx, inst, ctypes.byref(params), _stream(stream)))


def sae_get_params(ctx, inst, stream=None):
    p = SaeParams()
    _check(ctx, _lib.load().sae_get_params(ctx, inst, ctypes.byref(p), _stream(stream)))
    return p


def sae_get_counters(ctx, inst, stream=None):
    c = SaeCounters()
    _check(ctx, _lib.load().sae_get_counters(ctx, inst, ctypes.byref(c), _stream(stream)))
    return c


def sae_set_counters(ctx, inst, counters, stream=None):
    _check(ctx, _lib.load().sae_set_counters(ctx, inst, ctypes.byref(counters), _stream(stream)))


def sae_block_type(counts_u8, tau_u8, stream=None):
    n = counts_u8.shape[0]
    _check(None, _lib.load().sae_block_type(_ptr(counts_u8), n, _ptr(tau_u8), _stream(stream)))


FN_LN, FN_EXP, FN_ERFC = 0, 1, 2


def sae_recipe_eval(fn, x_f32, y_f32, stream=None):
    """The device realisation of ln / exp / erfc of the fp32 recipe, element-wise."""
    _check(None, _lib.load().sae_recipe_eval(int(fn), x_f32.numel(), _ptr(x_f32), _ptr(y_f32), _stream(stream)))


def sae_classify_blocks(ctx, hint_u8, meta_u16, roles, stream=None):
    """Algorithm 1 Classify on the device: rewrites the queue bits of meta."""
    r = (ctypes.c_int32 * 4)(*[int(x) for x in roles])
    _check(ctx, _lib.load().sae_classify_blocks(ctx, hint_u8.numel(), _ptr(hint_u8), _ptr(meta_u16), r,
                                                _stream(stream)))


def sae_index_build(ctx, stream=None):
    _check(ctx, _lib.load().sae_index_build(ctx, _stream(stream)))


def sae_insert_blocks(ctx, ids, hash, parent, last_access, meta, off, inst=None, stream=None):
    n = ids.numel()
    _check(ctx, _lib.load().sae_insert_blocks(ctx, n, _ptr(inst), _ptr(ids), _ptr(hash), _ptr(parent),
                                              _ptr(last_access), _ptr(meta), _ptr(off), _stream(stream)))


def sae_ref_blocks(ctx, ids, delta, inst=None, stream=None):
    _check(ctx, _lib.load().sae_ref_blocks(ctx, ids.numel(), _ptr(inst), _ptr(ids), int(delta), _stream(stream)))


def sae_prefix_match(ctx, hashes, lens, now, flags, match_len, matched_ids=None, inst=None, stream=None):
    n_req, max_len = hashes.shape
    _check(ctx, _lib.load().sae_prefix_match(ctx, n_req, max_len, _ptr(hashes), _ptr(lens), _ptr(inst), int(now),
                                             int(flags), _ptr(match_len), _ptr(matched_ids), _stream(stream)))


def sae_score_select(ctx, now, k, flags, victims, count, decision, decision_count, scores=None, k_per_inst=None,
                     stream=None):
    _check(ctx, _lib.load().sae_score_select(ctx, int(now), int(k), _ptr(k_per_inst), int(flags), _ptr(victims),
                                             _ptr(scores), _ptr(count), _ptr(decision), _ptr(decision_count),
                                             _stream(stream)))


def sae_match_select(ctx, hashes, lens, pm_now, pm_flags, match_len, now, k, flags, victims, count, decision,
                     decision_count, matched_ids=None, inst=None, scores=None, k_per_inst=None, stream=None):
    """sae_prefix_match then sae_score_select, as one call (same results)."""
    n_req, max_len = hashes.shape
    _check(ctx, _lib.load().sae_match_select(ctx, n_req, max_len, _ptr(hashes), _ptr(lens), _ptr(inst), int(pm_now),
                                             int(pm_flags), _ptr(match_len), _ptr(matched_ids), int(now), int(k),
                                             _ptr(k_per_inst), int(flags), _ptr(victims), _ptr(scores), _ptr(count),
                                             _ptr(decision), _ptr(decision_count), _stream(stream)))


def sae_feedback_update(ctx, flags=0, stream=None):
    _check(ctx, _lib.load().sae_feedback_update(ctx, int(flags), _stream(stream)))


def sae_poll_status(ctx, stream=None):
    b = ctypes.c_uint32()
    _check(ctx, _lib.load().sae_poll_status(ctx, _stream(stream), ctypes.byref(b)))
    return b.value


def sae_select_stats(ctx, inst, n_queues, stream=None):
    buf = (ctypes.c_uint32 * (4 * n_queues))()
    _check(ctx, _lib.load().sae_select_stats(ctx, inst, ctypes.cast(buf, ctypes.c_void_p), _stream(stream)))
    return [tuple(buf[4 * q:4 * q + 4]) for q in range(n_queues)]


def sae_profile_enable(ctx, enable=True):
    _check(ctx, _lib.load().sae_profile_enable(ctx, 1 if enable else 0))


def sae_profile_read(ctx):
    ms = ctypes.c_double()
    n = ctypes.c_int64()
    _check(ctx, _lib.load().sae_profile_read(ctx, ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


def sae_state_size(ctx):
    n = ctypes.c_size_t()
    _check(ctx, _lib.load().sae_state_size(ctx, ctypes.byref(n)))
    return n.value


def sae_save_state(ctx, inst, stream=None):
    """Instance `inst`'s context-held state as bytes (see include/sae.h)."""
    n = sae_state_size(ctx)
    buf = ctypes.create_string_buffer(n)
    _check(ctx, _lib.load().sae_save_state(ctx, inst, ctypes.cast(buf, ctypes.c_void_p), n, _stream(stream)))
    return buf.raw


def sae_load_state(ctx, inst, blob, stream=None):
    buf = ctypes.create_string_buffer(bytes(blob), len(blob))
    _check(ctx, _lib.load().sae_load_state(ctx, inst, ctypes.cast(buf, ctypes.c_void_p), len(blob),
                                           _stream(stream)))


def sae_get_intervals(ctx, inst, queue, cap=IVL_CAP, stream=None):
    """Algorithm 4's interval buffer of (inst, queue), oldest first (host list)."""
    buf = (ctypes.c_int32 * max(cap, 1))()
    n = ctypes.c_int32()
    _check(ctx, _lib.load().sae_get_intervals(ctx, inst, queue, ctypes.cast(buf, ctypes.c_void_p), cap,
                                              ctypes.byref(n), _stream(stream)))
    return list(buf[:min(n.value, cap)])


def sae_predict_sessions(h_bf16, w, work, logit, pred=None, stream=None):
    """Session predictor (Sec. 3.3) on n hidden states: h_bf16 is an int16
    tensor [n][d] of bf16 bit patterns; w holds device tensors w1 (int16
    [256][d], bf16 bits), b1, w2 [64][256], b2, w3 [64], b3 [1] (float32)."""
    n, d = h_bf16.shape
    p = SaePredictor()
    for name in ("w1", "b1", "w2", "b2", "w3", "b3"):
        setattr(p, name, _ptr(w[name]).value)
    _check(None, _lib.load().sae_predict_sessions(n, d, _ptr(h_bf16), ctypes.byref(p), _ptr(work), _ptr(logit),
                                                  _ptr(pred), _stream(stream)))


PRED_NOALLOC_MAX_N = 4096


def sae_predict_sessions_noalloc(h_bf16, w, logit, pred=None, stream=None):
    """As sae_predict_sessions, with the library's own per-GPU buffer in place
    of `work` (n <= PRED_NOALLOC_MAX_N); allocates nothing."""
    n, d = h_bf16.shape
    p = SaePredictor()
    for name in ("w1", "b1", "w2", "b2", "w3", "b3"):
        setattr(p, name, _ptr(w[name]).value)
    _check(None, _lib.load().sae_predict_sessions_noalloc(n, d, _ptr(h_bf16), ctypes.byref(p), _ptr(logit),
                                                          _ptr(pred), _stream(stream)))


# ------------------------------------------------- paged key-value cache
KV_BLOCK = 16
KV_BF16, KV_F16, KV_FP8 = 0, 1, 2
_KV_DTYPE = {torch.bfloat16: KV_BF16, torch.float16: KV_F16}
# what a cache's tensors may be, and its scales (bytes of an exponent)
_KV_HELD = {KV_BF16: (torch.bfloat16,), KV_F16: (torch.float16,), KV_FP8: (torch.uint8, torch.float8_e4m3fn)}
_KV_SCALES = (torch.uint8, torch.float8_e8m0fnu)


def _rows(t, heads, dim):
    """Data pointer, token stride and dtype of a [n][heads][dim] tensor of bf16 or f16 whose tokens may lie apart
    (a slice of fused rows); its heads and dimensions are contiguous."""
    if not t.is_cuda:
        raise SaeError("expected a device tensor")
    n, h, d = t.shape if t.dim() == 3 else (0, 0, 0)
    if h != heads or d != dim:
        raise SaeError("expected a tensor [n][%d][%d], got %s" % (heads, dim, tuple(t.shape)))
    s0, s1, s2 = t.stride()
    if n and (s2 != 1 or (s1 != dim and heads > 1)):
        raise SaeError("a token's heads must be contiguous")
    ty = _KV_DTYPE.get(t.dtype)
    if ty is None:
        raise SaeError("expected bfloat16 or float16")
    return t.data_ptr(), s0 if n > 1 else heads * dim, ty, n


def _same_device(what, tensors):
    """The device of the tensors (those that are not None)."""
    devices = {t.get_device() for t in tensors if t is not None}
    if len(devices) > 1:
        raise SaeError("%s are on different devices: %s" % (what, sorted(devices)))
    return devices.pop() if devices else None


def _raw_stream(kv, seqs, a, b, lse, work, stream):
    """The stream's handle, the current one by default, for a call on these tensors.  Launches go to the current device:
    everything has to be there.  (A decode step is a few microseconds: the handle is taken without making a stream, and
    the checks are written out.)"""
    here = torch._C._cuda_getDevice()
    if (a.get_device() != here or b.get_device() != here or (work is not None and work.get_device() != here) or
            (lse is not None and lse.get_device() != here) or kv.device not in (here, None) or
            seqs.device not in (here, None)):
        raise SaeError("a call's tensors must all be on the current device (%d)" % here)
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(here)
    if stream.device_index != here:
        raise SaeError("the stream must be on the current device (%d), it is on %d" % (here, stream.device_index))
    return stream.cuda_stream


def _check_blocks(name, t, blocks, stride, block):
    """A view with `blocks` blocks along its first dimension (or first ones) has them `stride` values apart, each of them
    `block` values in a row; a contiguous tensor of another shape is a buffer that holds them so."""
    n = lead = 1
    for lead, size in enumerate(t.shape[:-1], 1):
        n *= size
        if n >= blocks:
            break
    if t.is_contiguous() and (n != blocks or t.dim() < 2):
        return
    if t.dim() < 2 or n < blocks:
        raise SaeError("%s must be contiguous, or have the blocks along its first dimension" % name)
    apart = stride
    for i in range(lead - 1, -1, -1):
        if t.shape[i] > 1 and t.stride(i) != apart:
            raise SaeError("%s has its blocks %d values apart, not %d" % (name, t.stride(i), apart))
        apart *= t.shape[i]
    row = 1
    for size, step in zip(reversed(t.shape[lead:]), reversed(t.stride()[lead:])):
        if size > 1 and step != row:
            raise SaeError("a block of %s must be contiguous" % name)
        row *= size
    if row < block:
        raise SaeError("a block of %s must hold %d values" % (name, block))


def make_kv(type, n_instances, blocks_per_instance, n_kv_heads, head_dim, k, v, k_scale=None, v_scale=None, status=None,
            block_stride=0, scale_stride=0):
    """One layer's paged cache over device tensors (see sae_kv in include/sae.h); it keeps them alive.  k and v are
    of the cache's type (8-bit: uint8 or float8_e4m3fn) and of any shape, and hold the cache from their first element on:
    contiguous, or with block_stride (values; scale_stride, bytes) a view whose first dimension is the block."""
    kv = SaeKv()
    kv.type, kv.n_instances, kv.blocks_per_instance = int(type), int(n_instances), int(blocks_per_instance)
    kv.n_kv_heads, kv.head_dim = int(n_kv_heads), int(head_dim)
    kv.block_stride, kv.scale_stride = int(block_stride), int(scale_stride)
    if kv.type not in _KV_HELD:
        raise SaeError("unknown cache type")
    blocks = n_instances * blocks_per_instance

    def place(name, t, dtypes, stride, block):
        if t is None:
            return
        if not t.is_cuda:
            raise SaeError("expected a device tensor")
        if t.dtype not in dtypes:
            raise SaeError("%s must be %s for this type of cache" % (name, " or ".join(str(d)[6:] for d in dtypes)))
        size = t.element_size()
        if stride == 0 and not t.is_contiguous():
            raise SaeError("expected a contiguous tensor")
        if stride:
            _check_blocks(name, t, blocks, stride, block)
        need = ((blocks - 1) * (stride or block) + block) * size
        if t.untyped_storage().nbytes() - t.storage_offset() * size < need:
            raise SaeError("%s holds fewer than %d blocks" % (name, blocks))
        setattr(kv, name, t.data_ptr())
    place("k", k, _KV_HELD[kv.type], kv.block_stride, n_kv_heads * KV_BLOCK * head_dim)
    place("v", v, _KV_HELD[kv.type], kv.block_stride, n_kv_heads * KV_BLOCK * head_dim)
    place("k_scale", k_scale, _KV_SCALES, kv.scale_stride, n_kv_heads * KV_BLOCK)
    place("v_scale", v_scale, _KV_SCALES, kv.scale_stride, n_kv_heads * KV_BLOCK)
    if status is not None:
        if status.dtype not in (torch.int32, torch.uint32) or status.numel() < 1:
            raise SaeError("status must hold a 32-bit integer")
        kv.status = _ptr(status).value
    kv.tensors = (k, v, k_scale, v_scale, status)
    kv.device = _same_device("the cache's tensors", kv.tensors)
    return kv


def make_seqs(block_ids, kv_len, q_start=None, inst=None):
    """A call's sequences over device int32 tensors (see sae_seqs in include/sae.h); it keeps them alive.  block_ids
    [n][max_blocks] may be the matched_ids of sae_prefix_match."""
    n, width = block_ids.shape
    for name, t, count in (("block_ids", block_ids, n * width), ("kv_len", kv_len, n), ("q_start", q_start, n + 1),
                           ("inst", inst, n)):
        if t is not None and (t.dtype != torch.int32 or t.numel() != count):
            raise SaeError("%s must be int32 with %d elements" % (name, count))
    s = SaeSeqs()
    s.n_seq, s.max_blocks = n, width
    for name, t in (("block_ids", block_ids), ("kv_len", kv_len), ("q_start", q_start), ("inst", inst)):
        p = _ptr(t)
        setattr(s, name, p.value if p is not None else None)
    s.tensors = (block_ids, kv_len, q_start, inst)
    s.device = _same_device("the sequences' tensors", s.tensors)
    return s


def _kv_move(fn, kv, seqs, k, v, stream):
    heads, dim = kv.n_kv_heads, kv.head_dim
    kp, ks, kt, n = _rows(k, heads, dim)
    vp, vs, vt, vn = _rows(v, heads, dim)
    if kt != vt or n != vn:
        raise SaeError("k and v must have one type and one length")
    st = fn(ctypes.byref(kv), ctypes.byref(seqs), n, kt, kp, ks, vp, vs,
            _raw_stream(kv, seqs, k, v, None, None, stream))
    if st:
        _check(None, st)


def sae_kv_write(kv, seqs, k, v, stream=None):
    """Write the new tokens' keys and values [n][n_kv_heads][head_dim] (bf16 or f16) to their positions."""
    _kv_move(_lib.load().sae_kv_write, kv, seqs, k, v, stream)


def sae_kv_read(kv, seqs, k, v, stream=None):
    """Read the positions that sae_kv_write would write into k and v."""
    _kv_move(_lib.load().sae_kv_read, kv, seqs, k, v, stream)


def sae_attn_work_size(kv, seqs, n_tokens, n_heads):
    """Bytes of device scratch that an attention call of this size needs."""
    n = ctypes.c_size_t()
    _check(None, _lib.load().sae_attn_work_size(ctypes.byref(kv), ctypes.byref(seqs), int(n_tokens), int(n_heads),
                                                ctypes.byref(n)))
    return n.value


def _attn_rows(kv, q, out, lse, work):
    dim = kv.head_dim
    heads = q.shape[1] if q.dim() == 3 else 0
    qp, qs, qt, n = _rows(q, heads, dim)
    op, os_, ot, on = _rows(out, heads, dim)
    if ot != qt or on != n:
        raise SaeError("out must have q's type and shape")
    if lse is not None and (lse.dtype != torch.float32 or lse.numel() != n * heads):
        raise SaeError("lse must be float32 [n][heads]")
    return n, heads, qt, qp, qs, op, os_, _ptr(lse), _ptr(work), work.numel() * work.element_size()


def sae_attn_decode(kv, seqs, q, out, scale, work, window=0, lse=None, stream=None):
    """Attention of one new token per sequence: q, out [n_seq][heads][head_dim]."""
    n, heads, ty, qp, qs, op, os_, lp, wp, wn = _attn_rows(kv, q, out, lse, work)
    if n != seqs.n_seq:
        raise SaeError("q must have a row per sequence")
    st = _lib.load().sae_attn_decode(ctypes.byref(kv), ctypes.byref(seqs), heads, ty, qp, qs, op, os_, lp, scale,
                                     window, wp, wn, _raw_stream(kv, seqs, q, out, lse, work, stream))
    if st:
        _check(None, st)


def sae_attn_prefill(kv, seqs, q, out, scale, work, window=0, lse=None, stream=None):
    """Causal attention of the new tokens over their sequences' caches: q, out [n_tokens][heads][head_dim]."""
    n, heads, ty, qp, qs, op, os_, lp, wp, wn = _attn_rows(kv, q, out, lse, work)
    st = _lib.load().sae_attn_prefill(ctypes.byref(kv), ctypes.byref(seqs), n, heads, ty, qp, qs, op, os_, lp, scale,
                                      window, wp, wn, _raw_stream(kv, seqs, q, out, lse, work, stream))
    if st:
        _check(None, st)


TREE_MAX = 256


def sae_attn_tree(kv, seqs, parent, max_nodes, q, out, scale, work, window=0, lse=None, stream=None):
    """Attention of drafted tokens that form a tree per sequence over its cache and themselves: q, out
    [n_tokens][heads][head_dim], parent int32 [n_tokens] (see include/sae.h); no sequence has more than max_nodes."""
    n, heads, ty, qp, qs, op, os_, lp, wp, wn = _attn_rows(kv, q, out, lse, work)
    if parent.dtype != torch.int32 or parent.numel() != n:
        raise SaeError("parent must be int32 with %d elements" % n)
    pp = _ptr(parent)
    handle = _raw_stream(kv, seqs, q, out, lse, work, stream)
    if parent.get_device() != torch._C._cuda_getDevice():
        raise SaeError("a call's tensors must all be on the current device")
    st = _lib.load().sae_attn_tree(ctypes.byref(kv), ctypes.byref(seqs), n, pp, max_nodes, heads, ty, qp, qs, op, os_, lp,
                                   scale, window, wp, wn, handle)
    if st:
        _check(None, st)


def make_rope(inv_freq, interleaved=False, factor=1.0):
    """The position rotation of sae_kv_append: turns 2 len(inv_freq) dimensions of each head (see sae_rope in
    include/sae.h); it keeps the tensor alive."""
    if inv_freq.dtype != torch.float32:
        raise SaeError("inv_freq must be float32")
    r = SaeRope()
    r.inv_freq, r.factor = _ptr(inv_freq).value, float(factor)
    r.turned, r.interleaved = 2 * inv_freq.numel(), 1 if interleaved else 0
    r.tensors, r.device = (inv_freq,), inv_freq.get_device()
    return r


def sae_kv_append(kv, seqs, rope, q, q_out, k, v, pos=None, stream=None):
    """sae_kv_write with keys and queries [n_tokens][heads][head_dim] turned by their positions (pos int32 [n_tokens], or
    their places) on the way; the turned queries go to q_out, which may be q (both None: no queries)."""
    heads, dim = kv.n_kv_heads, kv.head_dim
    kp, ks, kt, n = _rows(k, heads, dim)
    vp, vs, vt, vn = _rows(v, heads, dim)
    if kt != vt or n != vn:
        raise SaeError("k and v must have one type and one length")
    qp = op = None
    qs = os_ = qh = 0
    if q is not None or q_out is not None:
        if q is None or q_out is None:
            raise SaeError("q and q_out go together")
        qh = q.shape[1] if q.dim() == 3 else 0
        qp, qs, qt, qn = _rows(q, qh, dim)
        op, os_, ot, on = _rows(q_out, qh, dim)
        if (qt, qn) != (kt, n) or (ot, on) != (kt, n):
            raise SaeError("q and q_out must have k's type and length")
    pp = None
    if pos is not None:
        if pos.dtype != torch.int32 or pos.numel() != n:
            raise SaeError("pos must be int32 with %d elements" % n)
        pp = _ptr(pos)
    handle = _raw_stream(kv, seqs, k, v, q, q_out, stream)
    here = torch._C._cuda_getDevice()
    if (pos is not None and pos.get_device() != here) or rope.device not in (here, None):
        raise SaeError("a call's tensors must all be on the current device (%d)" % here)
    st = _lib.load().sae_kv_append(ctypes.byref(kv), ctypes.byref(seqs), n, qh, kt, ctypes.byref(rope), pp, qp, qs, op, os_,
                                   kp, ks, vp, vs, handle)
    if st:
        _check(None, st)


# --------------------------------------------------------------- sampling
ROWS_F32 = 3
_LOGITS = {torch.bfloat16: KV_BF16, torch.float16: KV_F16, torch.float32: ROWS_F32}


def sae_sample_work_size(n_rows, vocab):
    """Bytes of device scratch that a sampling call of this size needs."""
    n = ctypes.c_size_t()
    _check(None, _lib.load().sae_sample_work_size(int(n_rows), int(vocab), ctypes.byref(n)))
    return n.value


def _vector(name, t, dtype, n, here):
    """Address of a row's settings or results, n values of `dtype` on the current device; None for none."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != n:
        raise SaeError("%s must be %s with %d elements" % (name, str(dtype)[6:], n))
    if t.get_device() != here:
        raise SaeError("a call's tensors must all be on the current device (%d)" % here)
    if not t.is_contiguous():
        raise SaeError("expected a contiguous tensor")
    return t.data_ptr()


def sae_sample(logits, u, token, work, temperature=None, top_k=None, top_p=None, min_p=None, prob=None, kept=None,
               stream=None):
    """A token per row of logits [n][vocab] (bf16, f16 or float32; rows may lie apart) from random numbers u [n] in [0, 1):
    token int32 [n].  temperature, top_p, min_p float32 and top_k int32, [n] each or None (see include/sae.h); prob float32
    and kept int32 [n] receive the token's share and the number of tokens that could be drawn."""
    if not logits.is_cuda:
        raise SaeError("expected a device tensor")
    ty = _LOGITS.get(logits.dtype)
    if ty is None or logits.dim() != 2:
        raise SaeError("logits must be [n][vocab] of bfloat16, float16 or float32")
    n, vocab = logits.shape
    stride, step = logits.stride()
    if n and vocab > 1 and step != 1:
        raise SaeError("a row of logits must be contiguous")
    here = torch._C._cuda_getDevice()
    if logits.get_device() != here or work.get_device() != here:
        raise SaeError("a call's tensors must all be on the current device (%d)" % here)
    f32, i32 = torch.float32, torch.int32
    settings = SaeSampling(_vector("temperature", temperature, f32, n, here), _vector("top_k", top_k, i32, n, here),
                           _vector("top_p", top_p, f32, n, here), _vector("min_p", min_p, f32, n, here))
    up, tp = _vector("u", u, f32, n, here), _vector("token", token, i32, n, here)
    pp, kp = _vector("prob", prob, f32, n, here), _vector("kept", kept, i32, n, here)
    if stream is None:
        handle = torch._C._cuda_getCurrentRawStream(here)
    elif stream.device_index != here:
        raise SaeError("the stream must be on the current device (%d), it is on %d" % (here, stream.device_index))
    else:
        handle = stream.cuda_stream
    st = _lib.load().sae_sample(n, vocab, ty, logits.data_ptr(), stride if n > 1 else vocab, settings, up, tp, pp, kp,
                                _ptr(work), work.numel() * work.element_size(), handle)
    if st:
        _check(None, st)


def status_names(bits):
    return [v for k, v in ST_NAMES.items() if bits & k]
