"""Device-buffer owners around the C ABI (allocation and marshalling only).

torch allocates device memory and supplies the stream; every computation
happens inside libdmtx.so.  Used by the tests, the smoke check and the
benchmark.
"""
from __future__ import annotations

from typing import Dict, Optional, Sequence

import torch

from . import lib
from .inputs import Shape, Workload

TORCH_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def desc_for(wl: Workload, layer: int = 0, **over) -> lib.LayerDesc:
    """Descriptor of a workload's layer; `plan=` names a lib.Plan."""
    kw = dict(layout=wl.layout, p_attn=wl.p_attn, p_attn_out=wl.p_attn_out, p_ffn_out=wl.p_ffn_out,
              seed=wl.seed, layer_id=layer, ln_eps=1e-12, self_attention=True)
    kw.update(over)
    return lib.make_desc(wl.shape, wl.dtype, **kw)


class EncoderLayer:
    """One encoder layer's device state: parameters, saved activations,
    workspace and fp32 gradients."""

    def __init__(self, desc: lib.LayerDesc, params: Dict[str, torch.Tensor], device="cuda",
                 workspace: Optional[torch.Tensor] = None):
        self.desc = desc
        self.device = torch.device(device)
        self.params = {n: t.to(self.device).contiguous() for n, t in params.items()}
        self.cparams = lib.make_params(self.params)
        self.saved_bytes, self.fwd_bytes, self.bwd_bytes = lib.encoder_layer_sizes(desc)
        self.saved = torch.empty(self.saved_bytes, dtype=torch.uint8, device=self.device)
        need = max(self.fwd_bytes, self.bwd_bytes)
        if workspace is None or workspace.numel() < need:
            workspace = torch.empty(need, dtype=torch.uint8, device=self.device)
        self.ws = workspace
        self.grads = {n: torch.empty(t.shape, dtype=torch.float32, device=self.device)
                      for n, t in self.params.items()}
        self.cgrads = lib.make_grads(self.grads)

    def forward(self, x: torch.Tensor, y: Optional[torch.Tensor] = None) -> torch.Tensor:
        if y is None:
            y = torch.empty_like(x)
        lib.encoder_layer_fwd(self.desc, self.cparams, x, y, self.saved, self.ws, self.ws.numel())
        return y

    def backward(self, x: torch.Tensor, dy: torch.Tensor, dx: Optional[torch.Tensor] = None) -> torch.Tensor:
        if dx is None:
            dx = torch.empty_like(x)
        lib.encoder_layer_bwd(self.desc, self.cparams, x, self.saved, dy, dx, self.cgrads, self.ws,
                              self.ws.numel())
        return dx

    def saved_tensor(self, name: str, shape, dtype) -> torch.Tensor:
        off, nbytes = lib.saved_tensor_view(self.desc, name)
        return self.saved[off:off + nbytes].view(dtype).view(*shape)


class MultiHeadAttention:
    """Attention-only device state (multi-head attention of Fig. 1a)."""

    def __init__(self, desc: lib.LayerDesc, params: Dict[str, torch.Tensor], device="cuda"):
        self.desc = desc
        self.device = torch.device(device)
        self.params = {n: t.to(self.device).contiguous() for n, t in params.items()}
        self.cparams = lib.make_params(self.params)
        self.saved_bytes, self.fwd_bytes, self.bwd_bytes = lib.mha_sizes(desc)
        self.saved = torch.empty(self.saved_bytes, dtype=torch.uint8, device=self.device)
        self.ws = torch.empty(max(self.fwd_bytes, self.bwd_bytes), dtype=torch.uint8, device=self.device)
        self.grads = {n: torch.empty(t.shape, dtype=torch.float32, device=self.device)
                      for n, t in self.params.items()}
        self.cgrads = lib.make_grads(self.grads)

    def forward(self, q, k=None, v=None, out=None):
        if out is None:
            out = torch.empty_like(q)
        lib.mha_fwd(self.desc, self.cparams, q, k, v, out, self.saved, self.ws, self.ws.numel())
        return out

    def backward(self, q, dout, k=None, v=None, dq=None, dk=None, dv=None):
        if dq is None:
            dq = torch.empty_like(q)
        if self.desc.self_attention != 1:
            dk = torch.empty_like(k) if dk is None else dk
        if self.desc.self_attention == 0:
            dv = torch.empty_like(v) if dv is None else dv
        lib.mha_bwd(self.desc, self.cparams, q, k, v, self.saved, dout, dq, dk, dv, self.cgrads, self.ws,
                    self.ws.numel())
        return dq, dk, dv


def _checked(name, t, dtype, shape, device):
    """A tensor's dtype, shape and device as the library will take them for granted."""
    if t.dtype != dtype or t.shape != shape or t.device != device:
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, expected {dtype} {tuple(shape)} on {device}")
    return t


def _dense(name, t, dtype, shape, device):
    if not _checked(name, t, dtype, shape, device).is_contiguous():
        raise ValueError(f"{name} is not contiguous")
    return t


def _launch(device, entry, *args):
    """An entry point on the device's current stream (and with the device as
    the current one, where it is not already); the stream's handle.  The
    library takes device pointers: host memory would be a fault of the kernels
    that read it."""
    if device.type != "cuda":
        raise ValueError(f"tensors on {device}: the kernels run on a GPU's")
    if device.index == torch.cuda.current_device():
        stream = torch.cuda.current_stream().cuda_stream
        entry(*args, stream=stream)
        return stream
    with torch.cuda.device(device):
        stream = torch.cuda.current_stream().cuda_stream
        entry(*args, stream=stream)
    return stream


def _apart(groups) -> None:
    """Contiguous tensors of {name: tensors} that are written by one call: no two share memory."""
    spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), n)
                   for n, ts in groups.items() if ts is not None for t in ts if t.numel())
    for (_, end, a), (begin, _, b) in zip(spans, spans[1:]):
        if begin < end:
            raise ValueError(f"{a} and {b}: two tensors share memory")


def _code(dtype: torch.dtype) -> int:
    for n, t in TORCH_DTYPES.items():
        if t == dtype:
            return lib.DTYPE_CODES[n]
    raise ValueError(f"unsupported dtype {dtype}")


class Attention:
    """Streaming attention (attn_fwd / attn_bwd) over tensors like q [B, J, H,
    P], k and v [B, K, G, P]: any strides with a contiguous last axis that
    are multiples of 8 elements.  Holds the descriptor, what the forward
    saves for the backward (train=True) and a workspace, so two calls of one
    object must not overlap.  Calls take tensors of the same shapes; a
    tensor with other strides gets a descriptor of its own for the call
    (gradients have their tensor's strides).

    q_len, k_len, prefix: int32 [B]; doc: int32 [B, K]; slopes: float32 [H];
    all on q's device, kept and read at every call.
    """

    def __init__(self, q, k, v, *, scaler: float = 0.0, cap: float = 0.0, causal: bool = False, q_len=None,
                 k_len=None, doc=None, prefix=None, slopes=None, train: bool = True):
        if q.dim() != 4 or k.dim() != 4:
            raise ValueError("q, k, v are [batch, tokens, heads, head size]")
        B, J, H, P = q.shape
        K, G = k.shape[1], k.shape[2]
        self.device, self.dtype, self.train = q.device, q.dtype, train
        self.shapes = {"q": (B, J, H, P), "k": (B, K, G, P), "v": (B, K, G, P), "out": (B, J, H, P)}
        self._aux = []
        for name, t, dt, shp in (("q_len", q_len, torch.int32, (B,)), ("k_len", k_len, torch.int32, (B,)),
                                 ("doc", doc, torch.int32, (B, K)), ("prefix", prefix, torch.int32, (B,)),
                                 ("slopes", slopes, torch.float32, (H,))):
            self._aux.append(None if t is None else _dense(name, t, dt, shp, self.device))
        d = lib.AttnDesc(B, J, K, H, G, P, _code(q.dtype), scaler, cap, 1 if causal else 0)
        d.q_len, d.k_len, d.doc, d.prefix, d.slopes = (lib.ptr(t) for t in self._aux)
        d.out = lib.AttnStride(J * H * P, P, H * P)
        self._strides = {"out": (J * H * P, H * P, P, 1)}
        self.desc = d
        for n, t in (("q", q), ("k", k), ("v", v)):
            self._take(n, t)
        self.saved_bytes, self.fwd_bytes, self.bwd_bytes = lib.attn_sizes(d)
        self.saved = torch.empty(self.saved_bytes, dtype=torch.uint8, device=self.device) if train else None
        self.ws_bytes = max(self.fwd_bytes, self.bwd_bytes if train else 0)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.device)

    def _take(self, name, t):
        """Checks a tensor and puts its strides into the descriptor."""
        s = t.stride()
        if t.dtype != self.dtype or t.shape != self.shapes[name] or t.device != self.device:
            _checked(name, t, self.dtype, self.shapes[name], self.device)
        if self._strides.get(name) != s:
            if s[3] != 1:
                raise ValueError(f"{name}: the last axis is not contiguous")
            # (the stride of an axis of one element is never taken: torch has any value there)
            b, j, h = (x if n > 1 else t.shape[3] for x, n in zip(s, t.shape[:3]))
            setattr(self.desc, name, lib.AttnStride(b, h, j))
            self._strides[name] = s

    def _like(self, name, t, of):
        """A gradient: shape and strides of its tensor."""
        _checked(name, t, self.dtype, of.shape, self.device)
        if any(n > 1 and a != b for n, a, b in zip(of.shape, t.stride(), of.stride())):
            raise ValueError(f"{name}: strides {t.stride()}, expected {of.stride()}")
        return t

    def _empty(self, of):
        return torch.empty_strided(of.shape, of.stride(), dtype=of.dtype, device=of.device)

    def forward(self, q, k, v, out=None):
        for n, t in (("q", q), ("k", k), ("v", v)):
            self._take(n, t)
        if out is None:
            out = torch.empty(self.shapes["out"], dtype=self.dtype, device=self.device)
        self._take("out", out)
        _launch(self.device, lib.attn_fwd, self.desc, q, k, v, out, self.saved, self.ws, self.ws_bytes)
        return out

    def backward(self, q, k, v, out, dout, dq=None, dk=None, dv=None):
        """(dq, dk, dv); out is the last forward's, dout has its strides."""
        if not self.train:
            raise ValueError("made with train=False: the forward saved nothing")
        for n, t in (("q", q), ("k", k), ("v", v), ("out", out)):
            self._take(n, t)
        self._like("dout", dout, out)
        dq = self._empty(q) if dq is None else self._like("dq", dq, q)
        dk = self._empty(k) if dk is None else self._like("dk", dk, k)
        dv = self._empty(v) if dv is None else self._like("dv", dv, v)
        _launch(self.device, lib.attn_bwd, self.desc, q, k, v, out, self.saved, dout, dq, dk, dv, self.ws,
                self.ws_bytes)
        return dq, dk, dv


class Embedding:
    """Embedding lookup and gradient (embed_fwd / embed_bwd): table [V, I],
    ids int32 of any shape, y ids.shape + [I], fp32 gradient [V, I].  The
    gradients of one object share its workspace and `grad`, captured ones
    too, so two of them must not overlap."""

    def __init__(self, table: torch.Tensor, scale: float = 1.0, pad_id: int = -1):
        if table.dim() != 2:
            raise ValueError("table is [vocabulary, width]")
        self.device, self.code = table.device, _code(table.dtype)
        self.table = _dense("table", table, table.dtype, table.shape, table.device)
        self.scale, self.pad_id = scale, pad_id
        self.grad = torch.empty(table.shape, dtype=torch.float32, device=table.device)
        self.ws = torch.empty(0, dtype=torch.uint8, device=table.device)
        self._used_on, self._captured = set(), False  # streams that used the workspace; whether a capture may have
        self._outgrown = []  # workspaces that captured backwards still use

    def forward(self, ids: torch.Tensor, y: Optional[torch.Tensor] = None) -> torch.Tensor:
        V, I = self.table.shape
        _dense("ids", ids, torch.int32, ids.shape, self.device)
        if y is None:
            y = torch.empty((*ids.shape, I), dtype=self.table.dtype, device=self.device)
        _dense("y", y, self.table.dtype, (*ids.shape, I), self.device)
        _launch(self.device, lib.embed_fwd, self.code, ids.numel(), V, I, ids, self.table, self.scale, y)
        return y

    def backward(self, ids: torch.Tensor, dy: torch.Tensor) -> torch.Tensor:
        """The table's gradient, in self.grad."""
        V, I = self.table.shape
        _dense("ids", ids, torch.int32, ids.shape, self.device)
        _dense("dy", dy, self.table.dtype, (*ids.shape, I), self.device)
        need = lib.embed_ws_bytes(ids.numel(), V, I)
        if self.ws.numel() < need:
            self._grow(need)
        stream = _launch(self.device, lib.embed_bwd, self.code, ids.numel(), V, I, ids, self.pad_id, dy, self.scale,
                         self.grad, self.ws, self.ws.numel())
        self._used_on.add(stream)
        # (the question is about the current device's stream)
        if torch.cuda.is_current_stream_capturing() or self.device.index != torch.cuda.current_device():
            self._captured = True
        return self.grad

    def _grow(self, need: int) -> None:
        """A larger workspace.  The one it replaces stays where a captured
        backward uses it; else its memory is free again once the streams it
        was used on have come so far."""
        if self._captured:
            self._outgrown.append(self.ws)
        else:
            for s in self._used_on:
                self.ws.record_stream(torch.cuda.ExternalStream(s, self.device))
        self.ws = torch.empty(max(need, 2 * self.ws.numel()), dtype=torch.uint8, device=self.device)
        self._used_on, self._captured = set(), False


STATE_BLOCK = 256  # elements of an 8-bit state that share a scale


class AdamW:
    """AdamW over a list of tensors (adamw_step).  params: contiguous tensors
    of one dtype; master: their fp32 copies ("auto": made here for 16-bit
    weights; None: none).  States are made here (zeros: before the first
    step) in fp32 or, with state_bits=8, as e4m3 codes with a scale for
    each 256 elements, unless given (m, v, and for 8 bits m_scale, v_scale:
    lists of flat tensors).  No two of all these share memory.  decay: one
    value or one for each tensor."""

    def __init__(self, params: Sequence[torch.Tensor], *, lr: float = 1e-3, beta1: float = 0.9, beta2: float = 0.999,
                 eps: float = 1e-8, decay=0.0, master="auto", state_bits: int = 32, m=None, v=None, m_scale=None,
                 v_scale=None):
        params = list(params)
        if not params:
            raise ValueError("no parameters")
        self.device, self.dtype = params[0].device, params[0].dtype
        if m is not None:
            state_bits = 32 if m[0].dtype == torch.float32 else 8
        self.params = [_dense("param", p, self.dtype, p.shape, self.device) for p in params]
        self._shapes = [p.shape for p in params]
        if isinstance(master, str):
            master = [p.float() for p in params] if self.dtype != torch.float32 else None
        sd = torch.float32 if state_bits == 32 else torch.float8_e4m3fn

        def states(name, given, dt, count):
            if given is None:
                # (zeros of the code's bytes: fill kernels of every type exist for uint8)
                given = [torch.zeros(count(p) * dt.itemsize, dtype=torch.uint8, device=self.device).view(dt)
                         for p in params]
            if len(given) != len(params):
                raise ValueError(f"{name}: {len(given)} tensors for {len(params)} parameters")
            return [_dense(name, t, dt, (count(p),), self.device) for t, p in zip(given, params)]

        def blocks(p):
            return -(-p.numel() // STATE_BLOCK)

        self.master = None if master is None else [_dense("master", t, torch.float32, p.shape, self.device)
                                                   for t, p in zip(master, params, strict=True)]
        self.m = states("m", m, sd, torch.Tensor.numel)
        self.v = states("v", v, sd, torch.Tensor.numel)
        self.m_scale = states("m_scale", m_scale, torch.float32, blocks) if state_bits == 8 else None
        self.v_scale = states("v_scale", v_scale, torch.float32, blocks) if state_bits == 8 else None
        _apart({"param": self.params, "master": self.master, "m": self.m, "v": self.v, "m_scale": self.m_scale,
                "v_scale": self.v_scale})
        decay = [float(decay)] * len(params) if isinstance(decay, (int, float)) else [float(x) for x in decay]
        none = [None] * len(params)
        rows = zip(self.params, self.master or none, none, self.m, self.v, self.m_scale or none, self.v_scale or none,
                   [p.numel() for p in params], decay, strict=True)
        self._items = (lib.AdamwTensor * len(params))(
            *[lib.AdamwTensor(*[lib.ptr(t) for t in r[:7]], *r[7:]) for r in rows])
        self.lr = lr
        self.desc = lib.AdamwDesc(_code(self.dtype), state_bits, lr, beta1, beta2, eps, 1.0, 0, None)

    def step(self, grads: Sequence[torch.Tensor], step: int, lr: Optional[float] = None, grad_scale: float = 1.0,
             scalars: Optional[torch.Tensor] = None) -> None:
        """Step number `step` (1 for the first) with fp32 gradients shaped like
        the parameters; lr: this step's, in place of self.lr.  scalars: float32 [4] on the device (see adamw_step),
        in place of step, lr and grad_scale."""
        if len(grads) != len(self.params):
            raise ValueError(f"{len(grads)} gradients for {len(self.params)} parameters")
        f32, dev = torch.float32, self.device
        for it, g, shape in zip(self._items, grads, self._shapes):
            if g.dtype != f32 or g.shape != shape or g.device != dev or not g.is_contiguous():
                _dense("grad", g, f32, shape, dev)
            it.grad = g.data_ptr()
        if scalars is not None:
            _dense("scalars", scalars, torch.float32, (4,), self.device)
        d = self.desc
        d.step, d.grad_scale, d.scalars = step, grad_scale, lib.ptr(scalars)
        d.lr = self.lr if lr is None else lr
        _launch(self.device, lib.adamw_step, d, self._items, len(self.params))
