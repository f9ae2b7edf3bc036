"""ctypes binding of libmsd.so (the C ABI declared in include/msd.h).

Argument marshalling only: every step of the decode path runs in the HIP
kernels of the library.  PyTorch supplies device memory and the stream.
If the library is missing this module raises -- there is no fallback.
"""
import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmsd.so")
MAX_TREE = 64

MSD_OK, MSD_ERR_INVALID_ARG, MSD_ERR_CAPACITY, MSD_ERR_STATE, MSD_ERR_HIP = 0, -1, -2, -3, -4
TREE_STATIC, TREE_DYNAMIC = 0, 1
F32, BF16, F16 = 0, 1, 2      # float types of the microscaled operators
MX_ROWS, MX_WEIGHT = 0, 1     # layouts of a quantised matrix

c_i32, c_f32, c_vp, c_sz = ctypes.c_int32, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t


class ModelDesc(ctypes.Structure):
    _fields_ = [("n_layers", c_i32), ("d_model", c_i32), ("n_heads", c_i32),
                ("n_kv_heads", c_i32), ("head_dim", c_i32), ("ffn_dim", c_i32),
                ("vocab", c_i32), ("rope_theta", c_f32), ("norm_eps", c_f32)]


class Limits(ctypes.Structure):
    _fields_ = [("max_batch", c_i32), ("max_seq", c_i32), ("max_tree", c_i32),
                ("max_prompt", c_i32)]


class LayerWeights(ctypes.Structure):
    _fields_ = [(n, c_vp) for n in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down",
                                    "attn_norm", "ffn_norm")]


class TargetWeights(ctypes.Structure):
    _fields_ = [("embed", c_vp), ("layers", ctypes.POINTER(LayerWeights)),
                ("final_norm", c_vp), ("lm_head", c_vp)]


class DraftWeights(ctypes.Structure):
    _fields_ = [("fc", c_vp), ("layer", LayerWeights)]


class Buffers(ctypes.Structure):
    _fields_ = [(n, c_vp) for n in ("target_k", "target_v", "draft_k", "draft_v", "workspace",
                                    "packed_weights")]


class TreeSpec(ctypes.Structure):
    _fields_ = [("kind", c_i32), ("n_nodes", c_i32), ("depth", c_i32), ("topk", c_i32),
                ("parent", ctypes.POINTER(c_i32)), ("rank", ctypes.POINTER(c_i32))]


class TraceRec(ctypes.Structure):
    _fields_ = [("kind", c_i32), ("m", c_i32), ("n", c_i32), ("k", c_i32), ("ms", c_f32)]


class Tree(ctypes.Structure):
    _fields_ = [("n_nodes", c_i32), ("token", c_i32 * MAX_TREE), ("parent", c_i32 * MAX_TREE),
                ("depth", c_i32 * MAX_TREE), ("score", c_f32 * MAX_TREE),
                ("anc", ctypes.c_uint64 * MAX_TREE)]


class Mx(ctypes.Structure):
    """A quantised matrix (msd_mx)."""
    _fields_ = [("codes_d", c_vp), ("scales_d", c_vp), ("rows", c_i32), ("cols", c_i32),
                ("layout", c_i32), ("terms", c_i32)]


class Sampling(ctypes.Structure):
    """Which tokens of a row of logits stay (msd_sampling)."""
    _fields_ = [("temperature", ctypes.c_double), ("top_p", ctypes.c_double),
                ("min_p", ctypes.c_double), ("top_k", c_i32)]

    def __init__(self, temperature=0.0, top_p=0.0, min_p=0.0, top_k=0):
        if not -1 << 31 <= top_k < 1 << 31:  # (ctypes would keep the low bits)
            raise ValueError(f"top_k: {top_k} does not fit 32 bits")
        super().__init__(temperature, top_p, min_p, top_k)


class Teacher(ctypes.Structure):
    """A teacher's top logits (msd_teacher)."""
    _fields_ = [("ids_d", c_vp), ("values_d", c_vp), ("k", c_i32),
                ("temperature", ctypes.c_double)]


_lib = None


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_2505_14260_amd/build.py")
        L = ctypes.CDLL(LIB_PATH)
        P = ctypes.POINTER
        L.msd_buffer_sizes.argtypes = [P(ModelDesc), P(Limits), P(c_sz), P(c_sz), P(c_sz), P(c_sz)]
        L.msd_create.argtypes = [P(ModelDesc), P(Limits), P(TargetWeights), P(DraftWeights),
                                 P(Buffers), c_vp, P(c_vp)]
        L.msd_workspace_size.argtypes = [P(ModelDesc), P(Limits), P(c_sz)]
        L.msd_destroy.argtypes = [c_vp]
        L.msd_last_error.argtypes = [c_vp]
        L.msd_last_error.restype = ctypes.c_char_p
        L.msd_prefill.argtypes = [c_vp, ctypes.c_int, ctypes.c_int, P(c_i32), P(ctypes.c_uint8),
                                  c_vp, P(c_i32)]
        L.msd_draft_tree.argtypes = [c_vp, ctypes.c_int, P(c_i32), P(TreeSpec), c_vp]
        L.msd_verify.argtypes = [c_vp, ctypes.c_int, P(c_i32), c_vp, ctypes.c_int, c_vp, c_vp]
        L.msd_verify_noalloc.argtypes = L.msd_verify.argtypes
        L.msd_accept_compact.argtypes = [c_vp, ctypes.c_int, P(c_i32), c_vp, ctypes.c_int, c_vp,
                                         P(c_i32), P(c_i32), c_vp]
        L.msd_accept_sample.argtypes = [c_vp, ctypes.c_int, P(c_i32), c_vp, ctypes.c_int, c_vp,
                                        ctypes.c_float, ctypes.c_uint64, P(c_i32), P(c_i32),
                                        c_vp]
        L.msd_seq_len.argtypes = [c_vp, ctypes.c_int]
        L.msd_set_state.argtypes = [c_vp, ctypes.c_int, ctypes.c_int, c_vp, c_i32]
        L.msd_set_draft_input.argtypes = [c_vp, ctypes.c_int]
        L.msd_use_caller_weights.argtypes = [c_vp, ctypes.c_int]
        L.msd_draft_mx_bytes.argtypes = [P(ModelDesc), P(c_sz)]
        L.msd_set_draft_mx.argtypes = [c_vp, c_vp]
        L.msd_stream_read.argtypes = [c_vp, c_sz, ctypes.c_int, c_vp, c_vp]
        L.msd_train_accumulate.argtypes = [c_vp, ctypes.c_int, ctypes.c_int, P(c_i32),
                                           P(ctypes.c_uint8), c_vp, P(ctypes.c_double)]
        L.msd_prefill_sample.argtypes = L.msd_prefill.argtypes[:-1] + [P(Sampling), c_f32, P(c_i32)]
        L.msd_train_record.argtypes = L.msd_train_accumulate.argtypes[:-1] + [ctypes.c_int, c_vp, c_vp,
                                                                              c_vp]
        L.msd_train_accumulate_top.argtypes = L.msd_train_accumulate.argtypes[:-1] + [
            P(Teacher), P(ctypes.c_double)]
        L.msd_train_apply.argtypes = [c_vp, ctypes.c_double]
        L.msd_train_read.argtypes = [c_vp, ctypes.c_int, c_vp, c_sz]
        L.msd_train_lr.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_double,
                                   P(ctypes.c_double)]
        L.msd_train_mix.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_int, P(c_i32), P(c_i32)]
        L.msd_mx_bytes.argtypes = [P(Mx), P(c_sz), P(c_sz)]
        L.msd_mx_quantize.argtypes = [c_vp, ctypes.c_int, c_sz, P(Mx), c_vp]
        L.msd_mx_dequantize.argtypes = [P(Mx), c_vp, ctypes.c_int, c_sz, c_vp]
        L.msd_mx_resid_norm.argtypes = [c_vp, c_sz, c_vp, c_sz, c_vp, c_sz, ctypes.c_int, c_vp,
                                        c_f32, P(Mx), c_vp]
        L.msd_mx_swiglu.argtypes = [c_vp, c_sz, c_vp, c_sz, ctypes.c_int, P(Mx), c_vp]
        L.msd_mx_product.argtypes = [P(Mx), P(Mx), c_vp, ctypes.c_int, c_sz, c_vp]
        rows = [c_vp, ctypes.c_int, c_sz, ctypes.c_int, ctypes.c_int]
        L.msd_logits_top.argtypes = rows + [ctypes.c_int, c_vp, c_vp, c_vp, c_vp]
        L.msd_logits_sample.argtypes = rows + [P(Sampling), c_vp, c_vp, c_vp, c_vp]
        L.msd_logits_filter.argtypes = rows + [P(Sampling), c_vp, c_sz, c_vp, c_vp]
        L.msd_logits_distill.argtypes = rows + [P(Teacher), c_vp, c_vp, c_vp, c_vp, c_sz, c_vp]
        L.msd_trace_enable.argtypes = [c_vp, ctypes.c_int, ctypes.c_int]
        L.msd_trace_read.argtypes = [c_vp, ctypes.c_int, P(TraceRec)]
        _lib = L
    return _lib


class MSDError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"msd error {code}: {msg}")
        self.code = code


def _check(ctx, rc):
    if rc != MSD_OK:
        msg = lib().msd_last_error(ctx)
        raise MSDError(rc, msg.decode() if msg else "")


def _i32(a):
    a = np.ascontiguousarray(a, dtype=np.int32)
    return a, a.ctypes.data_as(ctypes.POINTER(c_i32))


# --- the C entry points, same names -------------------------------------------------

def msd_buffer_sizes(desc: ModelDesc, lim: Limits):
    t, d, w, p = c_sz(), c_sz(), c_sz(), c_sz()
    _check(None, lib().msd_buffer_sizes(ctypes.byref(desc), ctypes.byref(lim), ctypes.byref(t),
                                        ctypes.byref(d), ctypes.byref(w), ctypes.byref(p)))
    return t.value, d.value, w.value, p.value


def msd_create(desc, lim, tw, dw, bufs, stream):
    out = c_vp()
    _check(None, lib().msd_create(ctypes.byref(desc), ctypes.byref(lim), ctypes.byref(tw),
                                  ctypes.byref(dw), ctypes.byref(bufs), stream, ctypes.byref(out)))
    return out.value


def msd_workspace_size(desc: ModelDesc, lim: Limits):
    w = c_sz()
    _check(None, lib().msd_workspace_size(ctypes.byref(desc), ctypes.byref(lim), ctypes.byref(w)))
    return w.value


def msd_destroy(ctx):
    _check(None, lib().msd_destroy(ctx))


def msd_last_error(ctx):
    m = lib().msd_last_error(ctx)
    return m.decode() if m else ""


def msd_prefill(ctx, seq, tokens, is_visual, visual_ptr):
    tok, ptok = _i32(tokens)
    vis = np.ascontiguousarray(is_visual, dtype=np.uint8)
    first = c_i32()
    _check(ctx, lib().msd_prefill(ctx, seq, len(tok), ptok,
                                  vis.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)),
                                  visual_ptr, ctypes.byref(first)))
    return first.value


def msd_prefill_sample(ctx, seq, tokens, is_visual, visual_ptr, how: Sampling, u):
    tok, ptok = _i32(tokens)
    vis = np.ascontiguousarray(is_visual, dtype=np.uint8)
    first = c_i32()
    _check(ctx, lib().msd_prefill_sample(ctx, seq, len(tok), ptok,
                                         vis.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)),
                                         visual_ptr, how, u, ctypes.byref(first)))
    return first.value


def msd_draft_tree(ctx, seqs, spec: TreeSpec, trees_ptr):
    s, ps = _i32(seqs)
    _check(ctx, lib().msd_draft_tree(ctx, len(s), ps, ctypes.byref(spec), trees_ptr))


def msd_verify(ctx, seqs, trees_ptr, n_nodes, argmax_ptr, logits_ptr=None):
    s, ps = _i32(seqs)
    _check(ctx, lib().msd_verify(ctx, len(s), ps, trees_ptr, n_nodes, argmax_ptr, logits_ptr))


def msd_verify_noalloc(ctx, seqs, trees_ptr, n_nodes, argmax_ptr, logits_ptr=None):
    s, ps = _i32(seqs)
    _check(ctx, lib().msd_verify_noalloc(ctx, len(s), ps, trees_ptr, n_nodes, argmax_ptr,
                                         logits_ptr))


def msd_accept_compact(ctx, seqs, trees_ptr, n_nodes, argmax_ptr, slot_map_ptr=None):
    s, ps = _i32(seqs)
    emitted = np.zeros((len(s), MAX_TREE), dtype=np.int32)
    n_emit = np.zeros(len(s), dtype=np.int32)
    _check(ctx, lib().msd_accept_compact(
        ctx, len(s), ps, trees_ptr, n_nodes, argmax_ptr,
        emitted.ctypes.data_as(ctypes.POINTER(c_i32)),
        n_emit.ctypes.data_as(ctypes.POINTER(c_i32)), slot_map_ptr))
    return [list(emitted[i, :n_emit[i]]) for i in range(len(s))]


def msd_accept_sample(ctx, seqs, trees_ptr, n_nodes, logits_ptr, temperature, seed,
                      slot_map_ptr=None):
    s, ps = _i32(seqs)
    emitted = np.zeros((len(s), MAX_TREE), dtype=np.int32)
    n_emit = np.zeros(len(s), dtype=np.int32)
    _check(ctx, lib().msd_accept_sample(
        ctx, len(s), ps, trees_ptr, n_nodes, logits_ptr, float(temperature), int(seed),
        emitted.ctypes.data_as(ctypes.POINTER(c_i32)),
        n_emit.ctypes.data_as(ctypes.POINTER(c_i32)), slot_map_ptr))
    return [list(emitted[i, :n_emit[i]]) for i in range(len(s))]


def msd_seq_len(ctx, seq):
    return lib().msd_seq_len(ctx, seq)


# draft input of visual prompt rows (msd_set_draft_input)
DRAFT_VISUAL_INPUTS = {"embedding": 0, "feature": 1}


def msd_set_draft_input(ctx, visual_input):
    _check(ctx, lib().msd_set_draft_input(ctx, visual_input))


def msd_use_caller_weights(ctx, enable):
    _check(ctx, lib().msd_use_caller_weights(ctx, 1 if enable else 0))


def msd_draft_mx_bytes(desc: ModelDesc):
    n = c_sz()
    _check(None, lib().msd_draft_mx_bytes(ctypes.byref(desc), ctypes.byref(n)))
    return n.value


def msd_set_draft_mx(ctx, weights_ptr):
    _check(ctx, lib().msd_set_draft_mx(ctx, weights_ptr))


def msd_train_accumulate(ctx, seq, tokens, is_visual, visual_ptr):
    """Loss sums (total, regression, token) of one training sequence; its
    gradient sums are added to the context's."""
    tok, ptok = _i32(tokens)
    vis = np.ascontiguousarray(is_visual, dtype=np.uint8)
    loss = (ctypes.c_double * 3)()
    _check(ctx, lib().msd_train_accumulate(ctx, seq, len(tok), ptok,
                                           vis.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)),
                                           visual_ptr, loss))
    return tuple(loss)


def msd_train_record(ctx, seq, tokens, is_visual, visual_ptr, k, values_ptr, ids_ptr, lse_ptr):
    tok, ptok = _i32(tokens)
    vis = np.ascontiguousarray(is_visual, dtype=np.uint8)
    _check(ctx, lib().msd_train_record(ctx, seq, len(tok), ptok,
                                       vis.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)),
                                       visual_ptr, k, values_ptr, ids_ptr, lse_ptr))


def msd_train_accumulate_top(ctx, seq, tokens, is_visual, visual_ptr, teacher: Teacher):
    """msd_train_accumulate with a teacher's record in place of the target's
    distribution."""
    tok, ptok = _i32(tokens)
    vis = np.ascontiguousarray(is_visual, dtype=np.uint8)
    loss = (ctypes.c_double * 3)()
    _check(ctx, lib().msd_train_accumulate_top(
        ctx, seq, len(tok), ptok, vis.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)), visual_ptr,
        teacher, loss))
    return tuple(loss)


def msd_train_apply(ctx, lr):
    _check(ctx, lib().msd_train_apply(ctx, lr))


def msd_train_read(ctx, what, out_ptr, n_floats):
    _check(ctx, lib().msd_train_read(ctx, what, out_ptr, n_floats))


def msd_train_lr(step, total_steps, lr_max):
    out = ctypes.c_double()
    _check(None, lib().msd_train_lr(step, total_steps, lr_max, ctypes.byref(out)))
    return out.value


def msd_train_mix(epoch, n_epochs, n_per_epoch):
    nt, nv = c_i32(), c_i32()
    _check(None, lib().msd_train_mix(epoch, n_epochs, n_per_epoch, ctypes.byref(nt),
                                     ctypes.byref(nv)))
    return nt.value, nv.value


def train_param_shapes(dims):
    """Shapes of the trained draft parameters in msd_train_read's order."""
    d, F = dims.d_model, dims.ffn_dim
    qd, kd = dims.n_heads * dims.head_dim, dims.n_kv_heads * dims.head_dim
    return [("fc", (d, 2 * d)), ("wq", (qd, d)), ("wk", (kd, d)), ("wv", (kd, d)),
            ("wo", (d, qd)), ("wg", (F, d)), ("wu", (F, d)), ("wd", (d, F)),
            ("attn_norm", (d,)), ("ffn_norm", (d,))]


def msd_set_state(ctx, seq, L, h_ptr, next_token):
    _check(ctx, lib().msd_set_state(ctx, seq, L, h_ptr, next_token))


def msd_stream_read(buf_ptr, nbytes, workgroups, sink_ptr, stream):
    _check(None, lib().msd_stream_read(buf_ptr, nbytes, workgroups, sink_ptr, stream))


def msd_mx_bytes(q: Mx):
    c, s = c_sz(), c_sz()
    _check(None, lib().msd_mx_bytes(q, ctypes.byref(c), ctypes.byref(s)))
    return c.value, s.value


def msd_mx_quantize(src_ptr, type_, ld, q: Mx, stream):
    _check(None, lib().msd_mx_quantize(src_ptr, type_, ld, q, stream))


def msd_mx_dequantize(q: Mx, dst_ptr, type_, ld, stream):
    _check(None, lib().msd_mx_dequantize(q, dst_ptr, type_, ld, stream))


def msd_mx_resid_norm(x_ptr, ldx, y_ptr, ldy, sum_ptr, lds, type_, gain_ptr, eps, q: Mx, stream):
    _check(None, lib().msd_mx_resid_norm(x_ptr, ldx, y_ptr, ldy, sum_ptr, lds, type_, gain_ptr,
                                         eps, q, stream))


def msd_mx_swiglu(gate_ptr, ldg, up_ptr, ldu, type_, q: Mx, stream):
    _check(None, lib().msd_mx_swiglu(gate_ptr, ldg, up_ptr, ldu, type_, q, stream))


def msd_mx_product(x: Mx, w: Mx, out_ptr, type_, ld, stream):
    _check(None, lib().msd_mx_product(x, w, out_ptr, type_, ld, stream))


def msd_logits_top(logits_ptr, type_, ld, rows, cols, k, values_ptr, ids_ptr, lse_ptr, stream):
    _check(None, lib().msd_logits_top(logits_ptr, type_, ld, rows, cols, k, values_ptr, ids_ptr,
                                      lse_ptr, stream))


def msd_logits_sample(logits_ptr, type_, ld, rows, cols, how: Sampling, uniforms_ptr, tokens_ptr,
                      logprobs_ptr, stream):
    _check(None, lib().msd_logits_sample(logits_ptr, type_, ld, rows, cols, how, uniforms_ptr,
                                         tokens_ptr, logprobs_ptr, stream))


def msd_logits_filter(logits_ptr, type_, ld, rows, cols, how: Sampling, out_ptr, ldo, kept_ptr,
                      stream):
    _check(None, lib().msd_logits_filter(logits_ptr, type_, ld, rows, cols, how, out_ptr, ldo,
                                         kept_ptr, stream))


def msd_logits_distill(logits_ptr, type_, ld, rows, cols, teacher: Teacher, loss_ptr, lse_ptr,
                       grad_ptr, dlogits_ptr, ldd, stream):
    _check(None, lib().msd_logits_distill(logits_ptr, type_, ld, rows, cols, teacher, loss_ptr,
                                          lse_ptr, grad_ptr, dlogits_ptr, ldd, stream))


def msd_trace_enable(ctx, capacity, kinds=0xF):
    _check(ctx, lib().msd_trace_enable(ctx, capacity, kinds))


def msd_trace_read(ctx, max_recs=4096):
    recs = (TraceRec * max_recs)()
    n = lib().msd_trace_read(ctx, max_recs, recs)
    if n < 0:
        _check(ctx, n)
    return [(r.kind, r.m, r.n, r.k, r.ms) for r in recs[:n]]


# --- convenience wrapper over device memory held in torch tensors --------------------

def make_static_spec(parent, rank):
    """parent/rank for nodes 1..N (root excluded), canonical order."""
    p, pp = _i32(parent)
    r, pr = _i32(rank)
    depth = np.zeros(len(p) + 1, dtype=np.int32)
    for i, q in enumerate(p, start=1):
        depth[i] = depth[q] + 1
    spec = TreeSpec(TREE_STATIC, len(p), int(depth.max()), 0, pp, pr)
    spec._keep = (p, r)
    return spec


def make_dynamic_spec(topk, depth, n_nodes):
    return TreeSpec(TREE_DYNAMIC, n_nodes, depth, topk, None, None)


def draw_uniform(seed, seq, length, j):
    """Draw j of the cycle of sequence slot `seq` that starts at a committed length
    (msd_accept_sample): a multiple of 2^-24 in [0, 1)."""
    mask = (1 << 64) - 1
    n = seq << 40 | length << 8 | j
    z = (seed + (n + 1) * 0x9E3779B97F4A7C15) & mask
    z = (z ^ z >> 30) * 0xBF58476D1CE4E5B9 & mask
    z = (z ^ z >> 27) * 0x94D049BB133111EB & mask
    return ((z ^ z >> 31) >> 40) / (1 << 24)


class Engine:
    """Owns device copies of the weights and the caller-side buffers."""

    def __init__(self, dims, target, draft, max_batch=1, max_seq=1024, max_tree=64,
                 max_prompt=1024, device="cuda", visual_input="embedding", draft_mx=False):
        import torch
        self.torch = torch
        self.dims = dims
        self.dev = torch.device(device)
        self._keep = []
        up = self._upload
        self.desc = ModelDesc(dims.n_layers, dims.d_model, dims.n_heads, dims.n_kv_heads,
                              dims.head_dim, dims.ffn_dim, dims.vocab, dims.rope_theta,
                              dims.norm_eps)
        self.lim = Limits(max_batch, max_seq, max_tree, max_prompt)
        layers = (LayerWeights * dims.n_layers)()
        for l, lw in enumerate(target["layers"]):
            layers[l] = self._layer(lw)
        self._layers = layers
        self.tw = TargetWeights(up(target["embed"]), layers, up(target["final_norm"]),
                                up(target["lm_head"]))
        self.dw = DraftWeights(up(draft["fc"]), self._layer(draft["layer"]))
        tkv, dkv, ws, pw = msd_buffer_sizes(self.desc, self.lim)
        self.bufs_t = [torch.empty(n, dtype=torch.uint8, device=self.dev)
                       for n in (tkv, tkv, dkv, dkv, ws, pw)]
        self.bufs = Buffers(*[b.data_ptr() for b in self.bufs_t])
        self.torch_stream = torch.cuda.current_stream(self.dev)
        self.stream = self.torch_stream.cuda_stream
        self.ctx = msd_create(self.desc, self.lim, self.tw, self.dw, self.bufs, self.stream)
        self.draft_mx = None
        self.set_draft_input(visual_input)
        if draft_mx:
            self.use_draft_mx()

    def set_draft_input(self, visual_input):
        """Draft input of the visual prompt rows of later prefills: "embedding"
        (the method) or "feature" (the Visual Feature variant)."""
        msd_set_draft_input(self.ctx, DRAFT_VISUAL_INPUTS[visual_input])

    def use_caller_weights(self, enable=True):
        """Training's target pass over more than 128 rows reads the row-major
        weights that this engine uploaded (and keeps) instead of unpacking the
        packed copies.  Same results."""
        msd_use_caller_weights(self.ctx, enable)

    def use_draft_mx(self, enable=True):
        """The draft in 4 bits (msd_set_draft_mx), in a buffer that this engine
        keeps, or back in bfloat16."""
        if not enable:
            msd_set_draft_mx(self.ctx, None)
            return
        if self.draft_mx is None:
            # on the engine's stream, which fills it: a block of the current stream may
            # still be in use there
            with self.torch.cuda.stream(self.torch_stream):
                self.draft_mx = self.torch.empty(msd_draft_mx_bytes(self.desc),
                                                 dtype=self.torch.uint8, device=self.dev)
        msd_set_draft_mx(self.ctx, self.draft_mx.data_ptr())

    def _visual(self, visual_bits):
        """Device copy of visual rows and its pointer (None for none)."""
        if visual_bits is None or not len(visual_bits):
            return None, None
        t = self.torch.from_numpy(np.ascontiguousarray(visual_bits).view(np.int16)).to(self.dev)
        return t, t.data_ptr()

    def train_accumulate(self, seq, tokens, is_visual, visual_bits, teacher=None):
        """Gradient sums of one training sequence; returns its loss sums.
        teacher: (ids, values, temperature), a record of the sequence's n - 1 rows as
        train_record() returns it, in place of the target's distribution."""
        vis_t, ptr = self._visual(visual_bits)
        if teacher is None:
            return msd_train_accumulate(self.ctx, seq, tokens, is_visual, ptr)
        torch = self.torch
        ids, values, temperature = teacher
        for t, dtype, what in ((ids, torch.int32, "ids"), (values, torch.float32, "values")):
            if t.dtype != dtype or t.dim() != 2 or t.shape[0] != len(tokens) - 1 \
                    or t.shape != ids.shape or not t.is_contiguous() \
                    or t.device != self.torch_stream.device:
                raise ValueError(f"teacher's {what}: wants contiguous {dtype} of {len(tokens) - 1} "
                                 f"rows on {self.torch_stream.device}, got {t.dtype} "
                                 f"{tuple(t.shape)} on {t.device}")
        self.torch_stream.wait_stream(torch.cuda.current_stream(self.dev))
        return msd_train_accumulate_top(
            self.ctx, seq, tokens, is_visual, ptr,
            Teacher(ids.data_ptr(), values.data_ptr(), ids.shape[1], temperature))

    def train_record(self, seq, tokens, is_visual, visual_bits, k):
        """The target's record of a training sequence for train_accumulate(): (ids, values)
        [n - 1, k] of its largest logits, on the engine's stream."""
        torch = self.torch
        vis_t, ptr = self._visual(visual_bits)
        shape = (max(len(tokens) - 1, 0), k)
        with torch.cuda.stream(self.torch_stream):
            ids = torch.empty(shape, dtype=torch.int32, device=self.dev)
            values = torch.empty(shape, dtype=torch.float32, device=self.dev)
        msd_train_record(self.ctx, seq, tokens, is_visual, ptr, k, values.data_ptr(),
                         ids.data_ptr(), None)
        current = torch.cuda.current_stream(self.dev)
        if current != self.torch_stream:
            current.wait_stream(self.torch_stream)
            ids.record_stream(current)
            values.record_stream(current)
        if vis_t is not None:
            vis_t.record_stream(self.torch_stream)
        return ids, values

    def train_apply(self, lr):
        msd_train_apply(self.ctx, lr)

    def train_read(self, what):
        """{name: float32 numpy array} of the gradient sums (what 0) or the
        master parameters (what 1)."""
        shapes = train_param_shapes(self.dims)
        n = sum(int(np.prod(s)) for _, s in shapes)
        buf = self.torch.empty(n, dtype=self.torch.float32, device=self.dev)
        msd_train_read(self.ctx, what, buf.data_ptr(), n)
        flat = buf.cpu().numpy()
        out, o = {}, 0
        for name, s in shapes:
            k = int(np.prod(s))
            out[name] = flat[o:o + k].reshape(s)
            o += k
        return out

    def _upload(self, a):
        a = np.ascontiguousarray(a)
        t = self.torch.from_numpy(a.view(np.int16)).to(self.dev)
        self._keep.append(t)
        return t.data_ptr()

    def _layer(self, lw):
        u = self._upload
        return LayerWeights(u(lw["wq"]), u(lw["wk"]), u(lw["wv"]), u(lw["wo"]), u(lw["wg"]),
                            u(lw["wu"]), u(lw["wd"]), u(lw["attn_norm"]), u(lw["ffn_norm"]))

    def close(self):
        if self.ctx:
            msd_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # views of the caller-owned KV caches (bf16 bits as int16)
    def kv_views(self):
        d = self.dims
        B, S, hd, KV = self.lim.max_batch, self.lim.max_seq, d.head_dim, d.n_kv_heads
        tk = self.bufs_t[0].view(self.torch.int16).view(d.n_layers, B, KV, S, hd)
        tv = self.bufs_t[1].view(self.torch.int16).view(d.n_layers, B, KV, hd, S)
        dk = self.bufs_t[2].view(self.torch.int16).view(1, B, KV, S, hd)
        dv = self.bufs_t[3].view(self.torch.int16).view(1, B, KV, hd, S)
        return tk, tv, dk, dv

    def prefill(self, seq, tokens, is_visual, visual_bits, sampling=None, u=0.0):
        """The first token of a prompt: the greedy one, or with a Sampling the one drawn
        with the uniform number u."""
        vis_t, ptr = self._visual(visual_bits)
        if sampling is not None:
            return msd_prefill_sample(self.ctx, seq, tokens, is_visual, ptr, sampling, u)
        return msd_prefill(self.ctx, seq, tokens, is_visual, ptr)

    def new_trees(self, n_seq):
        return self.torch.zeros(n_seq * ctypes.sizeof(Tree), dtype=self.torch.uint8, device=self.dev)

    @staticmethod
    def trees_to_host(trees_t, n_seq):
        raw = trees_t.cpu().numpy().tobytes()
        sz = ctypes.sizeof(Tree)
        return [Tree.from_buffer_copy(raw[i * sz:(i + 1) * sz]) for i in range(n_seq)]

    def draft_tree(self, seqs, spec, trees_t):
        msd_draft_tree(self.ctx, seqs, spec, trees_t.data_ptr())

    def verify(self, seqs, trees_t, n_nodes, want_logits=False):
        torch = self.torch
        amax = torch.empty(len(seqs) * n_nodes, dtype=torch.int32, device=self.dev)
        logits = None
        if want_logits:
            logits = torch.empty(len(seqs) * n_nodes, self.dims.vocab, dtype=torch.float32,
                                 device=self.dev)
        msd_verify(self.ctx, seqs, trees_t.data_ptr(), n_nodes, amax.data_ptr(),
                   logits.data_ptr() if logits is not None else None)
        return amax, logits

    def accept(self, seqs, trees_t, n_nodes, amax, want_slots=False):
        slots = None
        if want_slots:
            slots = self.torch.empty(len(seqs) * MAX_TREE, dtype=self.torch.int32, device=self.dev)
        em = msd_accept_compact(self.ctx, seqs, trees_t.data_ptr(), n_nodes, amax.data_ptr(),
                                slots.data_ptr() if slots is not None else None)
        return em, slots

    def accept_sample(self, seqs, trees_t, n_nodes, logits, temperature, seed,
                      want_slots=False, top_k=0, top_p=1.0, min_p=0.0):
        """Acceptance by speculative sampling; logits: verify's float32 logits.  With
        top_k, top_p or min_p the emitted tokens follow the target's distribution
        filtered by them (logits.filter)."""
        slots = None
        if top_k or top_p != 1.0 or min_p:
            from . import logits as ops
            with self.torch.cuda.stream(self.torch_stream):
                logits = ops.filter(logits, self.torch.empty_like(logits), temperature=temperature,
                                    top_k=top_k, top_p=top_p, min_p=min_p)
        if want_slots:
            slots = self.torch.empty(len(seqs) * MAX_TREE, dtype=self.torch.int32, device=self.dev)
        em = msd_accept_sample(self.ctx, seqs, trees_t.data_ptr(), n_nodes, logits.data_ptr(),
                               temperature, seed,
                               slots.data_ptr() if slots is not None else None)
        return em, slots

    def generate(self, seq, prompt, spec, n_new, record=False, temperature=0.0, seed=0,
                 top_k=0, top_p=1.0, min_p=0.0, sample_first=False):
        """Speculative decoding of one sequence: n_new tokens, greedy at
        temperature 0, else speculative sampling, from the distribution that
        top_k, top_p and min_p leave.  The first token, from the prompt, is the
        greedy one either way unless sample_first draws it too (with draw 255 of
        the cycle that starts at the prompt's length)."""
        tokens, is_visual, visual = prompt
        how = dict(top_k=top_k, top_p=top_p, min_p=min_p)
        if sample_first and temperature > 0:
            out = [self.prefill(seq, tokens, is_visual, visual,
                                Sampling(temperature, top_p, min_p, top_k),
                                draw_uniform(seed, seq, len(tokens), 255))]
        else:
            out = [self.prefill(seq, tokens, is_visual, visual)]
        T = spec.n_nodes + 1
        trees = self.new_trees(1)
        cycles = []
        while len(out) < n_new:
            self.draft_tree([seq], spec, trees)
            amax, logits = self.verify([seq], trees, T, want_logits=temperature > 0)
            if temperature > 0:
                em, _ = self.accept_sample([seq], trees, T, logits, temperature, seed, **how)
            else:
                em, _ = self.accept([seq], trees, T, amax)
            out.extend(int(t) for t in em[0])
            cycles.append(len(em[0]))
        return out[:n_new], cycles
