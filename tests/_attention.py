"""Attention with score modifiers in 64 bits, and how far a kernel that rounds
as the library states may be from it, element by element."""
import math

import torch

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
F = 2.0 ** -24  # a rounding in float32


def visible(B, J, K, causal=False, q_len=None, k_len=None, doc=None, prefix=None):
    """Truth of [B][J][K] from loops over the definition, and positions [B][J]."""
    see = torch.zeros(B, J, K, dtype=torch.bool)
    pos = torch.zeros(B, J, dtype=torch.int64)
    for b in range(B):
        nk = K if k_len is None else int(k_len[b])
        nq = J if q_len is None else int(q_len[b])
        for j in range(J):
            p = nk - nq + j
            pos[b, j] = p
            if j >= nq:
                continue
            row = torch.arange(K) < nk
            if causal:
                past = torch.arange(K) <= p
                if prefix is not None:
                    past |= torch.arange(K) < int(prefix[b])
                row &= past
            if doc is not None:
                mine = int(doc[b, p]) if 0 <= p < nk else -1
                row &= (doc[b] == mine) & (mine >= 0)
            see[b, j] = row
    return see, pos


def reference(q, k, v, dout=None, *, scaler=0.0, cap=0.0, causal=False, q_len=None, k_len=None, doc=None, prefix=None,
              slopes=None):
    """{name: (value, bound)} of out (and dq, dk, dv) for CPU tensors [B][L][heads][P]."""
    B, J, H, P = q.shape
    K, G = k.shape[1], k.shape[2]
    u = U[q.dtype]
    see, pos = visible(B, J, K, causal, q_len, k_len, doc, prefix)
    used_k = see.any(1)[:, :, None, None]
    used_q = see.any(2)[:, :, None, None]
    n = H // G
    scaler = scaler if scaler > 0 else 1 / math.sqrt(P)

    def heads(t, used, rep):  # what no query sees, or sees nothing, counts as zeros
        t = torch.where(used, t.double(), 0.0).permute(0, 2, 1, 3)
        return t.repeat_interleave(rep, 1)

    Q, Kh, V = heads(q, used_q, 1), heads(k, used_k, n), heads(v, used_k, n)
    raw = Q @ Kh.transpose(2, 3) * scaler
    size = Q.abs() @ Kh.abs().transpose(2, 3) * scaler
    # scores in float32: a product of P terms, then a few roundings of it
    ds = (P + 4) * F * size
    s, slope = raw, torch.ones_like(raw)
    if cap:
        t = torch.tanh(raw / cap)
        s, slope = cap * t, 1 - t * t
        ds = ds + cap * 8 * F  # the tanh itself: 4e-7 absolute
    if slopes is not None:
        far = (pos[:, None, :, None] - torch.arange(K)).abs().double()
        s = s - slopes.double()[None, :, None, None] * far
        ds = ds + 3 * F * slopes.double()[None, :, None, None] * far
    ds = ds + 6 * F * s.abs()
    m = see[:, None].expand(B, H, J, K)
    s = s.masked_fill(~m, float("-inf"))
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    e = torch.exp(s - top)
    l = e.sum(-1, keepdim=True)
    p = torch.where(l > 0, e / l.clamp_min(1e-300), 0.0)
    worst = torch.where(m, ds, 0.0).amax(-1, keepdim=True)
    dp_rel = 2 * (ds + worst) + (K + 16) * F  # relative error of a probability
    o = p @ V
    size_o = p @ V.abs()
    err_o = u * size_o + (p * dp_rel) @ V.abs() + (K + 8) * F * size_o
    out = {"out": (o, err_o * 1.01 + u * o.abs())}
    if q.dtype == torch.float16:  # values under the type's normal numbers
        out["out"] = (o, out["out"][1] + 2.0 ** -24 * (1 + V.abs().amax((2, 3), keepdim=True)))
    back = lambda t: t.permute(0, 2, 1, 3)  # noqa: E731
    if dout is not None:
        g = heads(dout, used_q, 1)
        dP = g @ V.transpose(2, 3)
        size_dP = g.abs() @ V.abs().transpose(2, 3)
        D = (g * o).sum(-1, keepdim=True)
        # D from the out of the forward, which has its error
        err_D = (g.abs() * (err_o + 2 * u * u * o.abs())).sum(-1, keepdim=True) + (P + 4) * F * (g * o).abs().sum(-1, keepdim=True)
        dc = p * (dP - D)
        err = p * ((P + 4) * F * size_dP + err_D) + (dp_rel + 4 * F) * p * ((dP - D).abs())
        dS = dc * slope
        err = err * slope + u * dS.abs() * 1.01 + (16 * F if cap else 0.0) * dc.abs()
        tiny = 0.0
        if q.dtype == torch.float16:
            # the score gradients' scale: their largest |dout|, to a power of two
            tiny = 2.0 ** -24 * g.abs().amax()
        err = torch.where(m, err + tiny, 0.0)
        ep = torch.where(m, u * p * 1.01 + dp_rel * p, 0.0)
        if q.dtype == torch.float16:
            ep = torch.where(m, ep + 2.0 ** -34, 0.0)

        def shared(t):
            return t.reshape(B, G, n, K, P).sum(2)

        dq, eq = dS @ Kh * scaler, err @ Kh.abs() * scaler
        dk, ek = shared(dS.transpose(2, 3) @ Q) * scaler, shared(err.transpose(2, 3) @ Q.abs()) * scaler
        dv, ev = shared(p.transpose(2, 3) @ g), shared(ep.transpose(2, 3) @ g.abs())
        sums = shared(dS.abs().transpose(2, 3) @ Q.abs()) * scaler, shared(p.transpose(2, 3) @ g.abs())
        eq = eq + (K + 8) * F * (dS.abs() @ Kh.abs()) * scaler
        ek, ev = ek + (n * J + 8) * F * sums[0], ev + (n * J + 8) * F * sums[1]
        for name, x, ex in (("dq", dq, eq), ("dk", dk, ek), ("dv", dv, ev)):
            ex = ex + u * x.abs() * 1.01
            if q.dtype == torch.float16:
                ex = ex + 2.0 ** -24
            out[name] = (x, ex)
    return {nme: (back(x), back(ex) + 1e-30) for nme, (x, ex) in out.items()}


def check(name, got, want):
    value, bound = want
    g = got.detach().cpu().double()
    assert g.shape == value.shape, (name, g.shape, value.shape)
    assert torch.isfinite(g).all(), f"{name}: not finite"
    ratio = (g - value).abs() / bound
    worst = float(ratio.max()) if ratio.numel() else 0.0
    at = [int(i) for i in torch.unravel_index(ratio.argmax(), ratio.shape)] if ratio.numel() else []
    assert worst <= 1.0, f"{name}: error {worst:.3g} times its bound at {at}: {g[tuple(at)]:.6g}, {value[tuple(at)]:.6g}"
    return worst
