"""Python binding of libosprey: the C-ABI calls under the same names, taking
torch tensors for device buffers.  Argument marshalling only -- every step of
the draft-and-verify path runs in the HIP kernels of the library.  PyTorch
provides device memory and the stream."""
from __future__ import annotations

import ctypes as C
from typing import Dict, Optional, Sequence

from . import _lib as L
from ._lib import osprey_config, osprey_layer_weights, osprey_weights  # noqa: F401

LAYER_FIELDS = ("in_norm", "w_qkv", "q_norm", "k_norm", "w_o", "post_norm", "w_gate", "w_up",
                "w_down")


class OspreyError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{L.STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


def _lib():
    return L.load()


def _check(rc: int) -> None:
    if rc != 0:
        raise OspreyError(rc, _lib().osprey_last_error().decode())


def _ptr(t) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


def _need(t, numel: int, dtype, name: str) -> None:
    """Refuse a device buffer that is smaller than the call will touch."""
    if t is None:
        return
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name}: need a contiguous device tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if t.numel() < numel:
        raise ValueError(f"{name}: {t.numel()} elements, the call needs {numel}")


def _i32_array(xs: Sequence[int]):
    arr = (C.c_int32 * len(xs))(*[int(x) for x in xs])
    return arr


def make_config(**kw) -> osprey_config:
    c = osprey_config()
    defaults = dict(n_taps=3, qk_norm=1, rms_eps=1e-6, rope_theta=1e6, kv_block=16, max_new_rows=1)
    for k, v in {**defaults, **kw}.items():
        setattr(c, k, v)
    return c


def config_validate(cfg: osprey_config) -> int:
    return int(_lib().osprey_config_validate(C.byref(cfg)))


def kv_bytes(cfg: osprey_config) -> int:
    return int(_lib().osprey_kv_bytes(C.byref(cfg)))


def workspace_bytes(cfg: osprey_config) -> int:
    return int(_lib().osprey_workspace_bytes(C.byref(cfg)))


def last_error() -> str:
    return _lib().osprey_last_error().decode()


def expected_weight_shapes(cfg) -> Dict[str, tuple]:
    """Shapes of the tensors include/osprey.h describes (osprey_weights)."""
    d, hd = cfg.d_model, cfg.head_dim
    s = {"embed": (cfg.vocab_target, d), "w_c": (d, cfg.n_taps * cfg.target_hidden),
         "final_norm": (d,), "lm_head": (cfg.vocab_draft, d)}
    for l in range(cfg.n_layers):
        p = f"layers.{l}."
        s.update({p + "in_norm": (d,), p + "w_qkv": ((cfg.n_q_heads + 2 * cfg.n_kv_heads) * hd, 2 * d),
                  p + "w_o": (d, cfg.n_q_heads * hd), p + "post_norm": (d,),
                  p + "w_gate": (cfg.d_ffn, d), p + "w_up": (cfg.d_ffn, d),
                  p + "w_down": (d, cfg.d_ffn)})
        if cfg.qk_norm:
            s.update({p + "q_norm": (hd,), p + "k_norm": (hd,)})
    return s


class Drafter:
    """A drafter handle plus the device buffers it was given.

    weights: name -> device tensor (dtype of the config), names as
    "embed", "w_c", "final_norm", "lm_head", "layers.{l}.{field}".
    d2t: int32 device tensor [V_d]."""

    def __init__(self, cfg: osprey_config, weights: Dict[str, "object"], d2t, stream=None):
        import torch
        self.cfg = cfg
        self.torch = torch
        _check(_lib().osprey_config_validate(C.byref(cfg)))
        dev = d2t.device
        want = torch.float32 if cfg.dtype == L.OSPREY_F32 else torch.bfloat16
        self._wdtype = want
        self.weights = {}
        for k, t in weights.items():
            if t.dtype != want or not t.is_contiguous() or t.device != dev:
                raise ValueError(f"weight {k}: need a contiguous {want} tensor on {dev}")
            self.weights[k] = t
        if d2t.dtype != torch.int32 or not d2t.is_contiguous() or d2t.numel() != cfg.vocab_draft:
            raise ValueError("d2t must be a contiguous int32 tensor of vocab_draft entries")
        shapes = expected_weight_shapes(cfg)
        for k, shp in shapes.items():
            if k not in self.weights:
                raise ValueError(f"missing weight {k}")
            if tuple(self.weights[k].shape) != shp:
                raise ValueError(f"weight {k}: shape {tuple(self.weights[k].shape)}, expected {shp}")
        self.d2t = d2t
        self.kv = torch.empty(kv_bytes(cfg), dtype=torch.uint8, device=dev)
        self.ws = torch.empty(workspace_bytes(cfg), dtype=torch.uint8, device=dev)
        self._layers = (osprey_layer_weights * cfg.n_layers)()
        for l in range(cfg.n_layers):
            for f in LAYER_FIELDS:
                t = self.weights.get(f"layers.{l}.{f}")
                setattr(self._layers[l], f, _ptr(t))
        self._w = osprey_weights(_ptr(self.weights["embed"]), _ptr(self.weights["w_c"]),
                                 _ptr(self.weights["final_norm"]), _ptr(self.weights["lm_head"]),
                                 _ptr(d2t), self._layers)
        self.stream = stream if stream is not None else torch.cuda.current_stream(dev)
        h = C.c_void_p()
        _check(_lib().osprey_draft_init(C.byref(cfg), C.byref(self._w), _ptr(self.kv),
                                        self.kv.numel(), _ptr(self.ws), self.ws.numel(),
                                        C.c_void_p(self.stream.cuda_stream), C.byref(h)))
        self.h = h
        self._keep = []

    # -- sequences --------------------------------------------------------------------
    def seq_reset(self, slot: int, block_ids: Sequence[int]) -> None:
        arr = _i32_array(block_ids)
        _check(_lib().osprey_seq_reset(self.h, slot, arr, len(block_ids)))

    def kv_append(self, slot: int, k, v) -> None:
        n = int(k.shape[1])
        c = self.cfg
        need = c.n_layers * n * c.n_kv_heads * c.head_dim
        _need(k, need, self._wdtype, "k")
        _need(v, need, self._wdtype, "v")
        _check(_lib().osprey_kv_append(self.h, slot, n, _ptr(k), _ptr(v)))

    def seq_truncate(self, slot: int, length: int) -> None:
        _check(_lib().osprey_seq_truncate(self.h, slot, length))

    def seq_length(self, slot: int) -> int:
        out = C.c_int32()
        _check(_lib().osprey_seq_length(self.h, slot, C.byref(out)))
        return int(out.value)

    # -- the step ---------------------------------------------------------------------
    def draft_step(self, slots, K: int, taps, temperature, u_draft=None, n_new=None,
                   new_tokens=None, taps_stride: int = 0, draft_tokens=None,
                   draft_logits=None, mask_token=None) -> None:
        """Ingest the new rows and propose K drafts: a chain of K steps
        (osprey_draft_step), or one block (osprey_draft_block) when mask_token is given."""
        torch, c = self.torch, self.cfg
        B = len(slots)
        tap_w = c.n_taps * c.target_hidden
        rows = B * taps_stride if taps_stride > 0 else int(sum(n_new or []))
        _need(taps, rows * tap_w, self._wdtype, "taps")
        _need(temperature, B, torch.float32, "temperature")
        _need(u_draft, B * K, torch.float32, "u_draft")
        _need(draft_tokens, B * K, torch.int32, "draft_tokens")
        _need(draft_logits, B * K * c.vocab_draft, torch.float32, "draft_logits")
        if n_new is not None:
            _need(new_tokens, int(sum(n_new)), torch.int32, "new_tokens")
        a, keep = _step_args(slots, K, taps, temperature, u_draft, n_new, new_tokens,
                             taps_stride, draft_tokens, draft_logits)
        if mask_token is None:
            _check(_lib().osprey_draft_step(self.h, C.byref(a)))
        else:
            _check(_lib().osprey_draft_block(self.h, C.byref(a), int(mask_token)))

    def draft_tree(self, slots, topk: int, depth: int, n_nodes: int, taps, temperature,
                   tokens, parents, n_new, new_tokens, taps_stride: int = 0,
                   scores=None) -> None:
        """Ingest the new rows and grow a draft tree (osprey_draft_tree); tokens and
        parents [B, n_nodes] int32 outputs, scores [B, n_nodes] float64 (optional)."""
        torch, c = self.torch, self.cfg
        B = len(slots)
        tap_w = c.n_taps * c.target_hidden
        rows = B * taps_stride if taps_stride > 0 else int(sum(n_new))
        _need(taps, rows * tap_w, self._wdtype, "taps")
        _need(temperature, B, torch.float32, "temperature")
        _need(new_tokens, int(sum(n_new)), torch.int32, "new_tokens")
        _need(tokens, B * n_nodes, torch.int32, "tokens")
        _need(parents, B * n_nodes, torch.int32, "parents")
        if scores is not None:
            _need(scores, B * n_nodes, torch.float64, "scores")
        a = L.osprey_step_args()
        a.batch = B
        a.K = 0
        sl = _i32_array(slots)
        a.slots = C.cast(sl, C.POINTER(C.c_int32))
        nn = _i32_array(n_new)
        a.n_new = C.cast(nn, C.POINTER(C.c_int32))
        a.new_tokens = _ptr(new_tokens)
        a.taps = _ptr(taps)
        a.taps_stride = taps_stride
        a.temperature = _ptr(temperature)
        t = L.osprey_tree_args()
        t.topk = topk
        t.depth = depth
        t.n_nodes = n_nodes
        t.tokens = _ptr(tokens)
        t.parents = _ptr(parents)
        t.scores = _ptr(scores) if scores is not None else None
        _check(_lib().osprey_draft_tree(self.h, C.byref(a), C.byref(t)))

    def verify(self, slots, K: int, target_logits, temperature, u_accept, u_bonus,
               accept_len, accept_mask, out_tokens, draft_temperature=None) -> None:
        torch, c = self.torch, self.cfg
        B = len(slots)
        _need(target_logits, B * (K + 1) * c.vocab_target, torch.float32, "target_logits")
        _need(temperature, B, torch.float32, "temperature")
        _need(u_accept, B * K, torch.float32, "u_accept")
        _need(u_bonus, B, torch.float32, "u_bonus")
        _need(accept_len, B, torch.int32, "accept_len")
        _need(accept_mask, B * K, torch.uint8, "accept_mask")
        _need(out_tokens, B * (K + 1), torch.int32, "out_tokens")
        _need(draft_temperature, B, torch.float32, "draft_temperature")
        a, keep = _verify_args(slots, K, target_logits, temperature, u_accept, u_bonus,
                               accept_len, accept_mask, out_tokens, draft_temperature)
        _check(_lib().osprey_verify(self.h, C.byref(a)))

    # -- one iteration as a HIP graph ---------------------------------------------------
    def set_stream(self, stream) -> None:
        """Enqueue subsequent calls on `stream` (a torch.cuda.Stream)."""
        _check(_lib().osprey_set_stream(self.h, C.c_void_p(stream.cuda_stream)))
        self.stream = stream

    def capture_iteration(self, slots, K: int, taps, draft_temperature, u_draft, draft_tokens,
                          draft_logits, target_logits, temperature, u_accept, u_bonus,
                          accept_len, accept_mask, out_tokens, max_context: int,
                          taps_stride: int, mask_token=None) -> "IterationGraph":
        """osprey_graph_capture: a pending-mode draft call and its verification recorded
        as one HIP graph over exactly these buffers (see IterationGraph)."""
        torch, c = self.torch, self.cfg
        B = len(slots)
        _need(taps, B * taps_stride * c.n_taps * c.target_hidden, self._wdtype, "taps")
        _need(draft_temperature, B, torch.float32, "draft_temperature")
        _need(u_draft, B * K, torch.float32, "u_draft")
        _need(draft_tokens, B * K, torch.int32, "draft_tokens")
        _need(draft_logits, B * K * c.vocab_draft, torch.float32, "draft_logits")
        _need(target_logits, B * (K + 1) * c.vocab_target, torch.float32, "target_logits")
        _need(temperature, B, torch.float32, "temperature")
        _need(u_accept, B * K, torch.float32, "u_accept")
        _need(u_bonus, B, torch.float32, "u_bonus")
        _need(accept_len, B, torch.int32, "accept_len")
        _need(accept_mask, B * K, torch.uint8, "accept_mask")
        _need(out_tokens, B * (K + 1), torch.int32, "out_tokens")
        sa, k1 = _step_args(slots, K, taps, draft_temperature, u_draft, None, None, taps_stride,
                            draft_tokens, draft_logits)
        va, k2 = _verify_args(slots, K, target_logits, temperature, u_accept, u_bonus,
                              accept_len, accept_mask, out_tokens, draft_temperature)
        g = C.c_void_p()
        _check(_lib().osprey_graph_capture(self.h, C.byref(sa),
                                           -1 if mask_token is None else int(mask_token),
                                           C.byref(va), int(max_context), C.byref(g)))
        # the graph holds raw pointers: keep the tensors alive with it
        return IterationGraph(self, g, (taps, draft_temperature, u_draft, draft_tokens,
                                        draft_logits, target_logits, temperature, u_accept,
                                        u_bonus, accept_len, accept_mask, out_tokens))

    def verify_rows(self, K: int, target_logits, draft_logits, draft_tokens, temperature,
                    u_accept, u_bonus, accept_len, accept_mask, out_tokens,
                    draft_temperature=None) -> None:
        torch, c = self.torch, self.cfg
        B = int(target_logits.shape[0])
        _need(target_logits, B * (K + 1) * c.vocab_target, torch.float32, "target_logits")
        _need(draft_logits, B * K * c.vocab_draft, torch.float32, "draft_logits")
        _need(draft_tokens, B * K, torch.int32, "draft_tokens")
        _need(temperature, B, torch.float32, "temperature")
        _need(u_accept, B * K, torch.float32, "u_accept")
        _need(u_bonus, B, torch.float32, "u_bonus")
        _need(accept_len, B, torch.int32, "accept_len")
        _need(accept_mask, B * K, torch.uint8, "accept_mask")
        _need(out_tokens, B * (K + 1), torch.int32, "out_tokens")
        _need(draft_temperature, B, torch.float32, "draft_temperature")
        a = L.osprey_verify_rows_args()
        a.batch = B
        a.K = K
        a.target_logits = _ptr(target_logits)
        a.draft_logits = _ptr(draft_logits)
        a.draft_tokens = _ptr(draft_tokens)
        a.temperature = _ptr(temperature)
        a.u_accept = _ptr(u_accept)
        a.u_bonus = _ptr(u_bonus)
        a.accept_len = _ptr(accept_len)
        a.accept_mask = _ptr(accept_mask)
        a.out_tokens = _ptr(out_tokens)
        a.draft_temperature = _ptr(draft_temperature)
        _check(_lib().osprey_verify_rows(self.h, C.byref(a)))

    def verify_tree(self, target_logits, tokens, parents, temperature, u_accept, u_bonus,
                    accept_len, accept_path, out_tokens) -> None:
        """Lossless verification of a draft tree (osprey_verify_tree): target_logits
        [B, N + 1, V_T], tokens / parents / u_accept [B, N], outputs accept_len [B],
        accept_path [B, N], out_tokens [B, N + 1]."""
        torch, c = self.torch, self.cfg
        B = int(target_logits.shape[0])
        N = int(target_logits.shape[1]) - 1
        _need(target_logits, B * (N + 1) * c.vocab_target, torch.float32, "target_logits")
        _need(tokens, B * N, torch.int32, "tokens")
        _need(parents, B * N, torch.int32, "parents")
        _need(temperature, B, torch.float32, "temperature")
        _need(u_accept, B * N, torch.float32, "u_accept")
        _need(u_bonus, B, torch.float32, "u_bonus")
        _need(accept_len, B, torch.int32, "accept_len")
        _need(accept_path, B * N, torch.int32, "accept_path")
        _need(out_tokens, B * (N + 1), torch.int32, "out_tokens")
        a = L.osprey_verify_tree_args()
        a.batch = B
        a.n_nodes = N
        a.target_logits = _ptr(target_logits)
        a.tokens = _ptr(tokens)
        a.parents = _ptr(parents)
        a.temperature = _ptr(temperature)
        a.u_accept = _ptr(u_accept)
        a.u_bonus = _ptr(u_bonus)
        a.accept_len = _ptr(accept_len)
        a.accept_path = _ptr(accept_path)
        a.out_tokens = _ptr(out_tokens)
        _check(_lib().osprey_verify_tree(self.h, C.byref(a)))

    # -- diagnostics ------------------------------------------------------------------
    def device_errors(self) -> int:
        f = C.c_uint32()
        _check(_lib().osprey_device_errors(self.h, C.byref(f)))
        return int(f.value)

    def kernel_timing(self, families=()) -> None:
        """Event timing of the given kernel families (KERNEL_*); () disables it."""
        mask = 0
        for f in families:
            mask |= 1 << int(f)
        _check(_lib().osprey_kernel_timing(self.h, mask))

    def kernel_time(self, family: int):
        ms, n = C.c_double(), C.c_int64()
        _check(_lib().osprey_kernel_time(self.h, family, C.byref(ms), C.byref(n)))
        return float(ms.value), int(n.value)

    def close(self) -> None:
        if getattr(self, "h", None):
            _lib().osprey_draft_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def verify_rows_static(K: int, target_logits, draft_logits, draft_tokens, temperature, u_accept,
                       u_bonus, accept_len, accept_mask, out_tokens, d2t, vocab_target: int,
                       stream=None, draft_temperature=None) -> None:
    """osprey_verify_rows_static: osprey_verify_rows with no handle; its scratch is the
    library's fixed device array (limits: batch 64, K 16, vocabularies 262144)."""
    import torch
    B = int(target_logits.shape[0])
    V_d = int(d2t.numel())
    _need(target_logits, B * (K + 1) * vocab_target, torch.float32, "target_logits")
    _need(draft_logits, B * K * V_d, torch.float32, "draft_logits")
    _need(draft_tokens, B * K, torch.int32, "draft_tokens")
    _need(temperature, B, torch.float32, "temperature")
    _need(u_accept, B * K, torch.float32, "u_accept")
    _need(u_bonus, B, torch.float32, "u_bonus")
    _need(accept_len, B, torch.int32, "accept_len")
    _need(accept_mask, B * K, torch.uint8, "accept_mask")
    _need(out_tokens, B * (K + 1), torch.int32, "out_tokens")
    _need(draft_temperature, B, torch.float32, "draft_temperature")
    _need(d2t, V_d, torch.int32, "d2t")
    a = L.osprey_verify_rows_args()
    a.batch = B
    a.K = K
    a.target_logits = _ptr(target_logits)
    a.draft_logits = _ptr(draft_logits)
    a.draft_tokens = _ptr(draft_tokens)
    a.temperature = _ptr(temperature)
    a.u_accept = _ptr(u_accept)
    a.u_bonus = _ptr(u_bonus)
    a.accept_len = _ptr(accept_len)
    a.accept_mask = _ptr(accept_mask)
    a.out_tokens = _ptr(out_tokens)
    a.draft_temperature = _ptr(draft_temperature)
    st = stream if stream is not None else torch.cuda.current_stream()
    _check(_lib().osprey_verify_rows_static(C.byref(a), _ptr(d2t), V_d, int(vocab_target),
                                            C.c_void_p(st.cuda_stream)))


# -- the 8-bit cache (osprey_kv8_*) --------------------------------------------------------

class Kv8Cache:
    """A paged key/value cache held in 8 bits (osprey_kv8_cache): codes uint8 [pages, 2,
    n_kv_heads, 16 * head_dim], scales float32 [pages, n_kv_heads, 2], page_table int32
    [batch, max_pages].  codes and scales may be strided over the pages (one layer of a pool);
    memory need not be cleared."""

    def __init__(self, codes, scales, page_table, head_dim: int):
        import torch
        if codes.dim() != 4 or codes.dtype != torch.uint8 or codes.shape[1] != 2 or codes.shape[3] != 16 * head_dim:
            raise ValueError(f"codes: need uint8 [pages, 2, n_kv_heads, {16 * head_dim}], got {codes.dtype} {tuple(codes.shape)}")
        pages, _, nkv, w = codes.shape
        if scales.dtype != torch.float32 or tuple(scales.shape) != (pages, nkv, 2):
            raise ValueError(f"scales: need float32 {(pages, nkv, 2)}, got {scales.dtype} {tuple(scales.shape)}")
        if page_table.dtype != torch.int32 or page_table.dim() != 2 or not page_table.is_contiguous():
            raise ValueError("page_table: need a contiguous int32 [batch, max_pages]")
        if codes.stride()[1:] != (nkv * w, w, 1) or scales.stride()[1:] != (2, 1):
            raise ValueError("codes and scales: a page must be contiguous")
        self.device = _same_device(codes, scales, page_table)
        self.codes, self.scales, self.page_table = codes, scales, page_table   # kept: the struct holds raw pointers
        self.batch, self.n_kv_heads, self.head_dim = int(page_table.shape[0]), nkv, head_dim
        # (one page: its stride is not used, and torch gives any)
        self.c = L.osprey_kv8_cache(_ptr(page_table), self.batch, int(page_table.shape[1]), pages, nkv, head_dim,
                                    _ptr(codes), codes.stride(0) if pages > 1 else 2 * nkv * w, _ptr(scales),
                                    scales.stride(0) if pages > 1 else 2 * nkv)
        self.ref = C.byref(self.c)


def _same_device(*tensors):
    dev = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != dev or dev < 0:
            raise ValueError(f"need tensors of one GPU, got {tensors[0].device} and {t.device}")
    return tensors[0].device


def _ints(t, numel: int, name: str):
    """The address of at least numel contiguous int32 (None: NULL)."""
    if t is None:
        return None
    if t.dtype is not _torch().int32 or not t.is_contiguous() or t.numel() < numel:
        raise ValueError(f"{name}: need {numel} contiguous int32, got {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def _heads(t, rows: int, hd: int, dtype, name: str) -> int:
    """The row stride of [rows, heads, hd] whose heads are contiguous."""
    sh = t.shape
    if len(sh) != 3 or t.dtype is not dtype or sh[0] != rows or sh[2] != hd:
        raise ValueError(f"{name}: need {dtype} [{rows}, heads, {hd}], got {t.dtype} {tuple(sh)}")
    st = t.stride()
    if st[2] != 1 or (st[1] != hd and sh[1] > 1):
        raise ValueError(f"{name}: the heads of a row must be contiguous")
    return st[0] if rows > 1 else sh[1] * hd


def _torch():
    import torch
    return torch


def _kv8_dtype(t) -> int:
    torch = _torch()
    if t.dtype is torch.bfloat16:
        return L.OSPREY_BF16
    if t.dtype is torch.float32:
        return L.OSPREY_F32
    raise ValueError(f"dtype {t.dtype}: need bfloat16 or float32")


def _kv8_call(fn, cache, a, stream) -> None:
    """Enqueue on `stream`, or the current stream of the cache's device, with that device current."""
    torch = _torch()
    st = stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(cache.device.index)
    if torch.cuda.current_device() == cache.device.index:
        rc = fn(cache.ref, C.byref(a), st)
    else:
        with torch.cuda.device(cache.device):
            rc = fn(cache.ref, C.byref(a), st)
    _check(rc)


def kv8_append(cache: Kv8Cache, k, v, cached, q=None, q_out=None, cu_rows=None, rope_pos=None, q_norm=None, k_norm=None,
               eps: float = 1e-6, rope_cos=None, rope_sin=None, errors=None, stream=None) -> None:
    """osprey_kv8_append: k, v [rows, n_kv_heads, head_dim] (rows may be strided: a slice of a
    QKV product) into the cache at positions cached[b] + j, and q [rows, n_q_heads, head_dim]
    into q_out, normalised per head where a gain is given and rotated where rope_cos / rope_sin
    [positions, head_dim / 2] are.  cu_rows int32 [batch + 1] groups the rows (None: one row
    per sequence).  errors: an int32 device word whose bits the kernels set."""
    rows, hd, dt = k.shape[0], cache.head_dim, k.dtype
    dtype = _kv8_dtype(k)
    _same_device(cache.codes, k, v, cached, q, q_out, cu_rows, rope_pos, q_norm, k_norm, rope_cos, rope_sin, errors)
    ks, vs, qs, os = _heads(k, rows, hd, dt, "k"), _heads(v, rows, hd, dt, "v"), 0, 0
    if k.shape[1] != cache.n_kv_heads or v.shape[1] != cache.n_kv_heads:
        raise ValueError(f"k and v: need {cache.n_kv_heads} heads")
    if q is not None:
        if q_out is None or q_out.shape != q.shape:
            raise ValueError("q_out: need a tensor of q's shape")
        qs, os = _heads(q, rows, hd, dt, "q"), _heads(q_out, rows, hd, dt, "q_out")
    for t, name in ((q_norm, "q_norm"), (k_norm, "k_norm")):
        if t is not None and (t.dtype is not dt or t.numel() != hd or not t.is_contiguous()):
            raise ValueError(f"{name}: need {hd} contiguous {dt}")
    if rope_cos is not None:
        for t in (rope_cos, rope_sin):
            if t is None or t.dtype is not _torch().float32 or t.dim() != 2 or t.shape[1] != hd // 2 or not t.is_contiguous() \
                    or t.shape != rope_cos.shape:
                raise ValueError(f"rope_cos and rope_sin: need contiguous float32 [positions, {hd // 2}] of one shape")
    a = L.osprey_kv8_append_args(
        rows, _ints(cu_rows, cache.batch + 1, "cu_rows"), _ints(cached, cache.batch, "cached"), _ints(rope_pos, rows, "rope_pos"), dtype,
        0 if q is None else q.shape[1], _ptr(q), k.data_ptr(), v.data_ptr(), qs, ks, vs, _ptr(q_norm), _ptr(k_norm), eps, _ptr(rope_cos),
        _ptr(rope_sin), 0 if rope_cos is None else rope_cos.shape[0], None if q is None else q_out.data_ptr(), os,
        _ints(errors, 1, "errors"))
    _kv8_call(_lib().osprey_kv8_append, cache, a, stream)


def kv8_attention_workspace(cache: Kv8Cache, rows: int, n_q_heads: int, max_rows: int, max_context: int) -> int:
    """Bytes of the workspace of a kv8_attention call with these sizes."""
    with _torch().cuda.device(cache.device):
        n = int(_lib().osprey_kv8_workspace_bytes(cache.ref, rows, n_q_heads, max_rows, max_context))
    if n == 0:
        raise OspreyError(L.OSPREY_E_INVALID, last_error())
    return n


def kv8_attention(cache: Kv8Cache, q, out, cached, workspace, max_rows: int = 1, max_context: int = 1, cu_rows=None,
                  scale=None, tree_mask=None, errors=None, stream=None) -> None:
    """osprey_kv8_attention: out [rows, n_q_heads, head_dim] = attention of q over what the rows
    see of the cache (their own positions already appended).  tree_mask int64 [rows, 2]: the
    bits of the new positions that a row sees.  max_rows, max_context: the largest row count and
    context the call is planned for.  workspace: uint8, kv8_attention_workspace bytes."""
    torch = _torch()
    rows, hd, dt = q.shape[0], cache.head_dim, q.dtype
    _same_device(cache.codes, q, out, cached, workspace, cu_rows, tree_mask, errors)
    if out.shape != q.shape:
        raise ValueError("out: need a tensor of q's shape")
    if tree_mask is not None and (tree_mask.dtype is not torch.int64 or tuple(tree_mask.shape) != (rows, 2) or not tree_mask.is_contiguous()):
        raise ValueError(f"tree_mask: need a contiguous int64 [{rows}, 2]")
    if workspace.dtype is not torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace: need a contiguous uint8 tensor")
    a = L.osprey_kv8_attention_args(
        rows, max_rows, max_context, _ints(cu_rows, cache.batch + 1, "cu_rows"), _ints(cached, cache.batch, "cached"), _ptr(tree_mask),
        _kv8_dtype(q), q.shape[1], q.data_ptr(), _heads(q, rows, hd, dt, "q"), hd ** -0.5 if scale is None else scale, out.data_ptr(),
        _heads(out, rows, hd, dt, "out"), workspace.data_ptr(), workspace.numel(), _ints(errors, 1, "errors"))
    _kv8_call(_lib().osprey_kv8_attention, cache, a, stream)


def kv8_keep(cache: Kv8Cache, base, path, n, errors=None, stream=None) -> None:
    """osprey_kv8_keep: position base[b] + i takes position base[b] + path[b, i], i < n[b]."""
    _same_device(cache.codes, base, path, n, errors)
    if path.dim() != 2 or path.shape[0] != cache.batch:
        raise ValueError(f"path: need [{cache.batch}, nodes]")
    a = L.osprey_kv8_keep_args(_ints(base, cache.batch, "base"), _ints(path, path.numel(), "path"), path.shape[1],
                               _ints(n, cache.batch, "n"), _ints(errors, 1, "errors"))
    _kv8_call(_lib().osprey_kv8_keep, cache, a, stream)


class IterationGraph:
    """A captured iteration (osprey_graph_*): launch() enqueues it on the drafter's
    stream; close() releases it (after the stream has finished with it)."""

    def __init__(self, drafter: Drafter, g, tensors):
        self.drafter, self.g, self._tensors = drafter, g, tensors

    def launch(self) -> None:
        _check(_lib().osprey_graph_launch(self.drafter.h, self.g))

    def close(self) -> None:
        if getattr(self, "g", None):
            _lib().osprey_graph_destroy(self.g)
            self.g = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _step_args(slots, K, taps, temperature, u_draft, n_new, new_tokens, taps_stride,
               draft_tokens, draft_logits):
    a = L.osprey_step_args()
    a.batch = len(slots)
    a.K = K
    sl = _i32_array(slots)
    a.slots = C.cast(sl, C.POINTER(C.c_int32))
    nn = None
    if n_new is not None:
        nn = _i32_array(n_new)
        a.n_new = C.cast(nn, C.POINTER(C.c_int32))
    a.new_tokens = _ptr(new_tokens)
    a.taps = _ptr(taps)
    a.taps_stride = taps_stride
    a.temperature = _ptr(temperature)
    a.u_draft = _ptr(u_draft)
    a.draft_tokens = _ptr(draft_tokens)
    a.draft_logits = _ptr(draft_logits)
    return a, (sl, nn)


def _verify_args(slots, K, target_logits, temperature, u_accept, u_bonus, accept_len,
                 accept_mask, out_tokens, draft_temperature):
    a = L.osprey_verify_args()
    a.batch = len(slots)
    a.K = K
    sl = _i32_array(slots)
    a.slots = C.cast(sl, C.POINTER(C.c_int32))
    a.target_logits = _ptr(target_logits)
    a.temperature = _ptr(temperature)
    a.u_accept = _ptr(u_accept)
    a.u_bonus = _ptr(u_bonus)
    a.accept_len = _ptr(accept_len)
    a.accept_mask = _ptr(accept_mask)
    a.out_tokens = _ptr(out_tokens)
    a.draft_temperature = _ptr(draft_temperature)
    return a, (sl,)


KERNEL_LM_HEAD, KERNEL_ATTENTION, KERNEL_VERIFY, KERNEL_DRAFT_STEP, KERNEL_QKV = range(5)
