"""What a program does with the library's operators around a layer, as cases.

Three kinds of pass, each through the public entry points or in its plain
form: attention over given projections (scores capped by a tanh, a bias that
falls with distance, documents, a prefix, ragged lengths, shared key/value
heads; a training step, a prompt's chunk, single tokens over a cache), the
embedding lookup with its gradient, and an AdamW step over many tensors.

Index letters: B batch, J query length, K key length, H heads, G key/value
heads, P head size, V vocabulary, I embedding width, F feed-forward width.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ cases
def _attn(name, do, dtype, B, J, K, H, G, P, causal=False, cap=0.0, alibi=False, doc=0, prefix=False, ragged=False):
    """doc: mean length of the documents packed into a sequence (0: one);
    prefix: each sequence's first quarter or so is seen by all its queries;
    ragged: sequences of different lengths, padded to K."""
    return dict(name=name, kind="attn", do=do, dtype=dtype, B=B, J=J, K=K, H=H, G=G, P=P, causal=causal, cap=cap,
                alibi=alibi, doc=doc, prefix=prefix, ragged=ragged)


def _embed(name, dtype, T, V, I):
    return dict(name=name, kind="embed", dtype=dtype, T=T, V=V, I=I)


def _adamw(name, dtype, bits, layers, I, F):
    return dict(name=name, kind="adamw", dtype=dtype, bits=bits, layers=layers, I=I, F=F)


def listed():
    return [
        # pre-training on packed documents: no query sees another document
        _attn("packed_bf16_step", "step", "bf16", 4, 4096, 4096, 16, 16, 64, doc=700),
        # a decoder layer with a distance bias, no tile divides the length
        _attn("alibi_f16_step", "step", "f16", 3, 1531, 1531, 12, 12, 64, causal=True, alibi=True),
        # one long sequence, capped scores, four query heads on a key/value head
        _attn("cap_bf16_step_long", "step", "bf16", 1, 8192, 8192, 16, 4, 128, causal=True, cap=30.0),
        # gradient checks of a small full-precision model: prefixes, ragged lengths
        _attn("prefix_f32_step", "step", "f32", 5, 203, 203, 4, 2, 32, causal=True, prefix=True, ragged=True),
        # serving: a prompt's chunk behind what the cache holds already
        _attn("chunk_bf16_fwd", "fwd", "bf16", 2, 500, 4096, 16, 8, 96, causal=True, ragged=True),
        # serving one user: the latency of one token
        _attn("one_f16_token", "fwd", "f16", 1, 1, 331, 12, 12, 64, causal=True),
        # serving a batch of users with long, different histories
        _attn("batch_bf16_token", "fwd", "bf16", 64, 1, 8192, 32, 4, 128, causal=True, ragged=True),
        # fine-tuning on one short sequence: the vocabulary's gradient is nearly all zeros
        _embed("embed_bf16_short", "bf16", 128, 30522, 768),
        # pre-training: 32 sequences of 512
        _embed("embed_f16_step", "f16", 16384, 30522, 1024),
        # a small full-precision layer's weights: all launch
        _adamw("adamw_f32_tiny", "f32", 32, 1, 32, 128),
        # a BERT-large layer, half-precision weights with fp32 master copies
        _adamw("adamw_f16_layer", "f16", 32, 1, 1024, 4096),
        # all layers of BERT-large, states in 8 bits
        _adamw("adamw_bf16_stack_8bit", "bf16", 8, 24, 1024, 4096),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _nameless(case):
    case.pop("name")
    return case


def draw(rng):
    what = rng.choice(["step", "step", "step", "step", "small", "chunk", "token", "token", "embed", "embed", "adamw",
                       "adamw"])
    if what == "embed":
        I = 8 * int(_log(rng, 8, 256))
        V = int(_log(rng, 100, 100000))
        return _nameless(_embed("", rng.choice(["bf16", "f16", "f32"]), int(_log(rng, 1, 65536 * 1024 / max(I, 1024))), V, I))
    if what == "adamw":
        I = 8 * int(_log(rng, 4, 128))
        layers = max(1, int(_log(rng, 1, 24)))
        return _nameless(_adamw("", rng.choice(["bf16", "f16", "f32"]), rng.choice([8, 32]), layers, I,
                                I * rng.choice([2, 3, 4])))
    dtype = rng.choice(["bf16", "f16"])
    G = rng.choice([1, 2, 4, 8])
    H = G * rng.choice([1, 1, 2, 4, 5])
    P = rng.choice([32, 64, 64, 64, 80, 96, 128, 128])
    kw = dict(causal=rng.random() < 0.6, cap=rng.choice([0.0, 0.0, 20.0, 50.0]), alibi=rng.random() < 0.3,
              ragged=rng.random() < 0.4)
    if what == "small":
        K = int(_log(rng, 2, 400))
        return _nameless(_attn("", "step", "f32", rng.randint(1, 6), K, K, H, G, rng.choice([8, 16, 32, 64, 128]),
                               prefix=kw["causal"] and rng.random() < 0.5, **kw))
    if what == "step":
        K = int(_log(rng, 33, 8192))
        B = max(1, int(_log(rng, 1, 2 ** 29 / (K * K * H) + 1)))
        if K * K * H > 2 ** 29:
            G, H = 1, max(1, 2 ** 29 // (K * K))
        doc = int(_log(rng, 8, K)) if rng.random() < 0.4 else 0
        return _nameless(_attn("", "step", dtype, min(B, 64), K, K, H, G if H % G == 0 else 1, P, doc=doc,
                               prefix=kw["causal"] and rng.random() < 0.3, **kw))
    kw["causal"] = True
    K = int(_log(rng, 16, 8192))
    if what == "chunk":
        return _nameless(_attn("", "fwd", dtype, rng.randint(1, 4), max(2, int(_log(rng, 2, min(K, 1024)))), K, H, G, P,
                               **kw))
    B = max(1, int(_log(rng, 1, min(64, 64 * 8192 / K))))
    return _nameless(_attn("", "fwd", dtype, B, 1, K, H, G, P, **kw))


# ------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _attn_inputs(c, seed):
    """q, k, v as a program has them: views of one fused projection in a
    training step, keys and values of a head-major cache when serving.
    Positions behind a sequence's length hold what was there before."""
    gen, dt = _generator(seed), TYPES[c["dtype"]]
    host = torch.Generator().manual_seed(int(seed))
    B, J, K, H, G, P = (c[n] for n in "BJKHGP")

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEV).to(dt)

    t = {}
    if c["do"] == "step":
        t["qkv"] = normal(B, K, H + 2 * G, P)
        t["q"], t["k"], t["v"] = t["qkv"][:, :, :H], t["qkv"][:, :, H:H + G], t["qkv"][:, :, H + G:]
        t["dout"] = normal(B, J, H, P)
    else:
        t["q"] = normal(B, J, H, P)
        t["k"], t["v"] = normal(B, G, K, P).transpose(1, 2), normal(B, G, K, P).transpose(1, 2)
    if c["ragged"]:
        low = min(K, J if c["do"] == "fwd" else max(1, K // 4))
        n = torch.randint(low, K + 1, (B,), generator=host)
        n[int(torch.randint(0, B, (1,), generator=host))] = K
        t["k_len"] = n.to(torch.int32).to(DEV)
        if c["do"] == "step":
            t["q_len"] = t["k_len"]
    if c["doc"]:
        D = c["doc"]
        cuts = torch.randint(max(1, D // 2), D + D // 2 + 1, (B, 2 * K // D + 3), generator=host).cumsum(1)
        t["doc"] = (torch.arange(K)[None, :, None] >= cuts[:, None, :]).sum(-1).to(torch.int32).to(DEV)
    if c["prefix"]:
        t["prefix"] = torch.randint(0, max(1, K // 2) + 1, (B,), generator=host).to(torch.int32).to(DEV)
    if c["alibi"]:
        t["slopes"] = torch.exp2(-8.0 * torch.arange(1, H + 1, dtype=torch.float64) / H).float().to(DEV)
    return t


def _embed_inputs(c, seed):
    """Ids are as frequent as words are: about uniform in the logarithm of
    the rank; the padding id takes a tenth of the places."""
    gen, dt = _generator(seed), TYPES[c["dtype"]]
    T, V, I = c["T"], c["V"], c["I"]
    u = torch.rand(T, generator=gen, device=DEV, dtype=torch.float64)
    ids = torch.exp(u * math.log(V)).long().clamp_(1, V - 1) if V > 1 else torch.zeros(T, dtype=torch.long, device=DEV)
    ids[torch.rand(T, generator=gen, device=DEV) < 0.1] = 0
    return {"ids": ids.to(torch.int32), "table": (torch.randn(V, I, generator=gen, device=DEV) * 0.02).to(dt),
            "dy": torch.randn(T, I, generator=gen, device=DEV).to(dt), "scale": math.sqrt(I)}


BLOCK = 256   # elements of an 8-bit state that share a scale
E4M3 = 448.0  # largest e4m3 value
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=100)


def _adamw_inputs(c, seed):
    """All layers' tensors in flat buffers, each at a multiple of the state
    block, as a data-parallel program keeps them: weights in the storage type
    and in fp32, fp32 gradients, states after a hundred steps."""
    gen, dt = _generator(seed), TYPES[c["dtype"]]
    I, F = c["I"], c["F"]
    matrices = [I * I] * 4 + [F * I] * 2
    vectors = [I] * 4 + [I] * 4 + [F] + [I]
    sizes = (matrices + vectors) * c["layers"]
    at, n = [], 0
    for s in sizes:
        at.append(n)
        n += -(-s // BLOCK) * BLOCK
    width = (-(-torch.tensor(sizes) // BLOCK) * BLOCK).to(DEV)
    decays = ([0.01] * len(matrices) + [0.0] * len(vectors)) * c["layers"]
    decay = torch.tensor(decays, dtype=torch.float64).to(DEV)
    inside = torch.zeros(n + 1, dtype=torch.int32)
    inside.index_add_(0, torch.tensor(at), torch.ones(len(at), dtype=torch.int32))
    inside.index_add_(0, torch.tensor(at) + torch.tensor(sizes), -torch.ones(len(at), dtype=torch.int32))
    inside = inside.cumsum(0)[:n].bool().to(DEV)

    def normal(std):
        return torch.where(inside, torch.randn(n, generator=gen, device=DEV) * std, 0.0)

    master = normal(0.02)
    m, r = normal(1e-3), normal(5e-3).abs()
    t = {"sizes": sizes, "at": at, "decays": decays, "decay": decay, "width": width, "n": n,
         "grad": normal(1e-2)}
    t["param"] = master.to(dt)
    if c["dtype"] != "f32":
        t["master"] = master
    else:
        t["param"] = master
    if c["bits"] == 32:
        t["m"], t["v"] = m, r * r
    else:
        t["m"], t["m_scale"] = _pack(m, False)
        t["v"], t["v_scale"] = _pack(r, True)
    return t


INPUTS = {"attn": _attn_inputs, "embed": _embed_inputs, "adamw": _adamw_inputs}


def prepare(case, seed):
    s = {"case": case, **INPUTS[case["kind"]](case, seed)}
    if own:
        from paper_2007_00072_amd import runner
        if case["kind"] == "attn":
            s["attention"] = runner.Attention(s["q"], s["k"], s["v"], **_modifiers(s))
        elif case["kind"] == "embed":
            s["embedding"] = runner.Embedding(s["table"], scale=s["scale"], pad_id=0)
        else:
            views = {k: [s[k][a:a + n] for a, n in zip(s["at"], s["sizes"])] if k in s else None
                     for k in ("param", "grad", "master", "m", "v")}
            for k in ("m_scale", "v_scale"):
                views[k] = [s[k][a // BLOCK:(a + n + BLOCK - 1) // BLOCK] for a, n in zip(s["at"], s["sizes"])] \
                    if k in s else None
            h = HYPER
            s["optimizer"] = runner.AdamW(views["param"], master=views["master"], m=views["m"], v=views["v"],
                                          m_scale=views["m_scale"], v_scale=views["v_scale"],
                                          decay=s["decays"], lr=h["lr"], beta1=h["beta1"], beta2=h["beta2"],
                                          eps=h["eps"])
            s["grads"] = views["grad"]
    return s


def _modifiers(s):
    c = s["case"]
    return dict(causal=c["causal"], cap=c["cap"], train=c["do"] == "step",
                **{n: s.get(n) for n in ("q_len", "k_len", "doc", "prefix", "slopes")})


# ------------------------------------------------------------------ passes
def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"attn": _own_attn, "embed": _own_embed, "adamw": _own_adamw}[kind](state)
    return {"attn": _plain_attn, "embed": _plain_embed, "adamw": _plain_adamw}[kind](state)


def _own_attn(s):
    a = s["attention"]
    out = a.forward(s["q"], s["k"], s["v"])
    if s["case"]["do"] == "fwd":
        return {"out": out}
    H, G = s["case"]["H"], s["case"]["G"]
    dqkv = torch.empty_like(s["qkv"])
    a.backward(s["q"], s["k"], s["v"], out, s["dout"], dqkv[:, :, :H], dqkv[:, :, H:H + G], dqkv[:, :, H + G:])
    return {"out": out, "dqkv": dqkv}


def _own_embed(s):
    e = s["embedding"]
    return {"y": e.forward(s["ids"]), "dtable": e.backward(s["ids"], s["dy"])}


def _own_adamw(s):
    s["optimizer"].step(s["grads"], HYPER["step"])
    return _states(s, s["m"], s["v"])


def _states(s, m, v):
    """Every buffer the step updated; 8-bit states as their e4m3 values, with the scales."""
    names = [n for n in ("param", "master", "m_scale", "v_scale") if n in s]
    return {"m": m, "v": v, **{n: s[n] for n in names}}


def _visible(s):
    """[B][1][J][K]: which keys a query sees; and [B][J] positions of the queries."""
    c = s["case"]
    B, J, K = c["B"], c["J"], c["K"]
    key = torch.arange(K, device=DEV)
    k_len = s["k_len"].long() if "k_len" in s else torch.full((B,), K, device=DEV)
    q_len = s["q_len"].long() if "q_len" in s else torch.full((B,), J, device=DEV)
    row = torch.arange(J, device=DEV)
    pos = (k_len - q_len)[:, None] + row
    see = (key < k_len[:, None])[:, None, :] & (row < q_len[:, None])[:, :, None]
    if c["causal"]:
        past = key <= pos[:, :, None]
        if "prefix" in s:
            past = past | (key < s["prefix"].long()[:, None])[:, None, :]
        see = see & past
    if "doc" in s:
        mine = torch.gather(s["doc"].long(), 1, pos.clamp(0, K - 1))
        see = see & (mine[:, :, None] == s["doc"][:, None, :]) & (pos >= 0)[:, :, None]
    return see[:, None], pos


def _plain_attn(s):
    c = s["case"]
    B, J, K, H, G, P = (c[n] for n in "BJKHGP")
    dt, scaler = TYPES[c["dtype"]], 1.0 / math.sqrt(P)

    def heads(t, n):  # [B][L][n heads][P] -> [B][G][n / G * L][P]
        return t.float().permute(0, 2, 1, 3).reshape(B, G, -1, P)

    q, k, v = heads(s["q"], H), heads(s["k"], G), heads(s["v"], G)
    see, pos = _visible(s)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).view(B, H, J, K) * scaler
    slope = None
    if c["cap"]:
        x = torch.tanh(x / c["cap"])
        if c["do"] == "step":
            slope = 1 - x * x
        x = x * c["cap"]
    if "slopes" in s:
        far = (pos[:, :, None] - torch.arange(K, device=DEV)).abs().float()
        x = x - s["slopes"][:, None, None] * far[:, None]
    x = x.masked_fill(~see, float("-inf"))
    top = x.amax(-1, keepdim=True).clamp_min(-1e30)
    x = torch.exp(x - top)
    p = x / x.sum(-1, keepdim=True).clamp_min(1e-30)
    o = torch.matmul(p.view(B, G, -1, K), v)
    out = o.view(B, H, J, P).permute(0, 2, 1, 3).to(dt).contiguous()
    if c["do"] == "fwd":
        return {"out": out}
    live = see.any(-1).to(torch.float32)[:, :, :, None]  # rows without a key hold zeros
    g = (s["dout"].float().permute(0, 2, 1, 3) * live).reshape(B, G, -1, P)
    dv = torch.matmul(p.view(B, G, -1, K).transpose(2, 3).contiguous(), g)
    dx = torch.matmul(g, v.transpose(2, 3).contiguous()) - (g * o).sum(-1, keepdim=True)
    dx = dx.view(B, H, J, K) * p * scaler
    if slope is not None:
        dx = dx * slope
    dx = dx.view(B, G, -1, K)
    dq = torch.matmul(dx, k)
    dk = torch.matmul(dx.transpose(2, 3).contiguous(), q)
    parts = (dq.view(B, H, J, P), dk.view(B, G, K, P), dv.view(B, G, K, P))
    return {"out": out, "dqkv": torch.cat([t.permute(0, 2, 1, 3) for t in parts], 2).to(dt)}


def _plain_embed(s):
    c, ids = s["case"], s["ids"].long()
    y = (s["table"][ids].float() * s["scale"]).to(TYPES[c["dtype"]])
    dtable = torch.zeros(c["V"], c["I"], device=DEV)
    dtable.index_add_(0, ids, s["dy"].float())
    dtable *= s["scale"]
    dtable[0] = 0
    return {"y": y, "dtable": dtable}


def _pack(x, root):
    """Blocks of 256 as e4m3 values of x / scale with scale = max |x| / 448;
    for roots (the second moment's), what is not zero stays above zero."""
    top = x.view(-1, BLOCK).abs().amax(1)
    held = top >= 2.0 ** -100
    scale = torch.where(held, top / E4M3, 0.0)
    code = x.view(-1, BLOCK) * torch.where(held, E4M3 / top, 0.0)[:, None]
    code = code.to(torch.float8_e4m3fn)
    if root:
        code = torch.where((x.view(-1, BLOCK) > 0) & (code.float() == 0), 2.0 ** -9, code.float()).to(torch.float8_e4m3fn)
    return code.view(-1), scale


def _plain_adamw(s):
    c, h = s["case"], HYPER
    b1, b2 = h["beta1"], h["beta2"]
    keep = torch.repeat_interleave((1.0 - h["lr"] * s["decay"]).float(), s["width"], output_size=s["n"])
    g = s["grad"]
    w = s["master"] if "master" in s else s["param"]
    if c["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m = (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        r = (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1)
        v = r * r
    m = m * b1 + g * (1.0 - b1)
    v = v * b2 + (g * g) * (1.0 - b2)
    u = (m * (1.0 / (1.0 - b1 ** h["step"]))) / (torch.sqrt(v * (1.0 / (1.0 - b2 ** h["step"]))) + h["eps"])
    w.copy_(w * keep - u * h["lr"])
    if "master" in s:
        s["param"].copy_(w)
    if c["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        for n, x in (("m", m), ("v", torch.sqrt(v))):
            code, scale = _pack(x, n == "v")
            s[n].copy_(code)
            s[n + "_scale"].copy_(scale)
    return _states(s, s["m"], s["v"])


# ------------------------------------------------------------------ work
def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "embed":
        # ids, the rows looked up, y; dy and the whole fp32 gradient
        return {"bytes": 8 * c["T"] + es * c["T"] * c["I"] * 3 + 4 * c["V"] * c["I"], "flops": 2 * c["T"] * c["I"]}
    if c["kind"] == "adamw":
        n = c["layers"] * (4 * c["I"] ** 2 + 2 * c["I"] * c["F"] + 9 * c["I"] + c["F"])
        states = 16 if c["bits"] == 32 else 4 + 16 / BLOCK
        return {"bytes": n * (4 + 8 + (0 if es == 4 else es) + states), "flops": 15 * n}
    B, J, K, H, G, P = (c[n] for n in "BJKHGP")
    # lengths are about uniform between the shortest and K
    low = J if c["do"] == "fwd" else max(1, K // 4)
    L = (low + K) / 2 if c["ragged"] and B > 1 else K
    rows = min(J, L)
    span = L  # keys a query sees
    if c["causal"]:
        span = L - (rows - 1) / 2
        if c["prefix"]:
            span += L / 24  # a prefix of 0 to half the keys
    if c["doc"]:
        span = min(span, c["doc"] * (0.55 if c["causal"] else 1.09))
    pairs = B * H * rows * span
    io = B * (2 * rows * H * P + 2 * L * G * P)
    if c["do"] == "fwd":
        return {"bytes": es * io, "flops": 4 * P * pairs}
    return {"bytes": es * (2 * io + 2 * B * rows * H * P), "flops": (4 + 10) * P * pairs}


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    t = INPUTS[case["kind"]](case, seed)
    return {"attn": _exact_attn, "embed": _exact_embed, "adamw": _exact_adamw}[case["kind"]](case, t)


def _exact_attn(c, t):
    """One sequence and key/value head at a time, the gradients by
    differentiation of the forward."""
    B, J, K, H, G, P = (c[n] for n in "BJKHGP")
    step, n = c["do"] == "step", c["H"] // c["G"]
    out = torch.zeros(B, J, H, P, dtype=torch.float64, device=DEV)
    grads = torch.zeros(B, K, H + 2 * G, P, dtype=torch.float64, device=DEV) if step else None
    for b in range(B):
        nk = int(t["k_len"][b]) if "k_len" in t else K
        nq = int(t["q_len"][b]) if "q_len" in t else J
        if nk == 0 or nq == 0:
            continue
        p, k_at = torch.arange(nq, device=DEV) + (nk - nq), torch.arange(nk, device=DEV)
        hidden = torch.zeros(nq, nk, dtype=torch.bool, device=DEV)
        if c["causal"]:
            hidden |= k_at[None, :] > p[:, None]
            if "prefix" in t:
                hidden[:, :int(t["prefix"][b])] = False
        if "doc" in t:
            ids = t["doc"][b, :nk]
            hidden |= ids[p][:, None] != ids[None, :]
        for g in range(G):
            k = t["k"][b, :nk, g].double().requires_grad_(step)
            v = t["v"][b, :nk, g].double().requires_grad_(step)
            for h in range(g * n, g * n + n):
                q = t["q"][b, :nq, h].double().requires_grad_(step)
                with torch.set_grad_enabled(step):
                    a = q @ k.t() / math.sqrt(P)
                    if c["cap"]:
                        a = c["cap"] * torch.tanh(a / c["cap"])
                    if "slopes" in t:
                        a = a - t["slopes"][h].double() * (p[:, None] - k_at[None, :]).abs()
                    y = torch.softmax(a.masked_fill(hidden, float("-inf")), -1) @ v
                out[b, :nq, h] = y.detach()
                if step:
                    y.backward(t["dout"][b, :nq, h].double())
                    grads[b, :nq, h] = q.grad
                del a, y
            if step:
                grads[b, :nk, H + g], grads[b, :nk, H + G + g] = k.grad, v.grad
    return {"out": out, "dqkv": grads} if step else {"out": out}


def _exact_embed(c, t):
    ids = t["ids"].long()
    d = torch.zeros(c["V"], c["I"], dtype=torch.float64, device=DEV)
    used = ids != 0
    d.index_add_(0, ids[used], t["dy"][used].double())
    return {"y": t["table"][ids].double() * t["scale"], "dtable": d * t["scale"]}


def _exact_adamw(c, t):
    h = HYPER
    decay = torch.repeat_interleave(t["decay"], t["width"])
    g = t["grad"].double()
    w = t["master" if "master" in t else "param"].double()
    if c["bits"] == 32:
        m, v = t["m"].double(), t["v"].double()
    else:
        m = (t["m"].double().view(-1, BLOCK) * t["m_scale"].double()[:, None]).view(-1)
        v = (t["v"].double().view(-1, BLOCK) * t["v_scale"].double()[:, None]).view(-1) ** 2
    m += (1 - h["beta1"]) * (g - m)
    v += (1 - h["beta2"]) * (g * g - v)
    root = torch.sqrt(v / (1 - h["beta2"] ** h["step"]))
    w -= h["lr"] * (decay * w + m / (1 - h["beta1"] ** h["step"]) / (root + h["eps"]))
    out = {"param": w}
    if "master" in t:
        out["master"] = w
    if c["bits"] == 32:
        return {"m": m, "v": v, **out}
    for n, x in (("m", m), ("v", torch.sqrt(v))):
        blocks = x.view(-1, BLOCK)
        top = blocks.abs().amax(1, keepdim=True)
        e = blocks / (top / E4M3).clamp_min(1e-300)
        # e4m3: three bits behind the leading one down to 2^-6, steps of 2^-9 below
        step = torch.exp2(torch.floor(torch.log2(e.abs().clamp_min(2.0 ** -6))) - 3)
        code = torch.round(e / step) * step
        if n == "v":
            code = torch.where((blocks > 0) & (code == 0), 2.0 ** -9, code)
        out[n], out[n + "_scale"] = code.view(-1), top[:, 0] / E4M3
    return out
