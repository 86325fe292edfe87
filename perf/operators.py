"""What the operators around the expert pool are timed on: the norm in front of a layer, the balance loss over sequences, the
pool's experts in 8 bits, and the layout of weights in 8 bits.

A case is a dict of plain values:
  op        "norm": residual added, root-mean-square norm, and its backward pass (training);
            "norm_mx8": the same norm forward only, with its output in 8 bits beside the one the router reads (serving);
            "balance": balance loss over the sequences of a batch, with its gradient;
            "experts": the pool's experts on 8-bit rows with 8-bit weights (serving);
            "quantize": a matrix to 8 bits with scales
  dtype     "bf16" or "f32", of the activations (or of the matrix)
  T, d      tokens, d_model ("quantize": rows and columns);  f, E, k as in the expert pool
  residual  "norm", "norm_mx8": whether a residual is added
  n_seq, padded   "balance": sequences of ragged lengths, some of them empty; whether rows behind the last one belong to none
  router    "balance": "norm" or "softmax";  skew  "experts", "balance": "none" or "hot"

8 bits: e4m3 values with a scale 2^e for every 32 neighbours of a row, e the smallest integer >= -127 for which the largest of them
is at most 448 * 2^e; scales are bytes e + 127, four bytes of a row and 128 columns together: [ceil(columns / 128)][rows][4].
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
NORM_EPS = 1e-6
EPS = 1e-6
SIGMA = 1.1
C = 2.5
ALPHA = 2e-2
WEIGHT_STD = 0.02


def _case(name=None, **kw):
    c = dict(op="norm", dtype="bf16", T=128, d=64, f=64, E=1, k=1, residual=True, n_seq=1, padded=False, router="norm", skew="none")
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # float mode as a reference run of a reduced model with a ragged width, trained
        _case("norm-train-reduced-f32", dtype="f32", T=1001, d=252),
        # the largest training configuration: the norm in front of one of its layers
        _case("norm-train-largest", T=32768, d=1536),
        # serving: one sequence decoding a token, and a prompt of about 4000 tokens
        _case("norm-8bit-one-token", op="norm_mx8", T=1, d=1536),
        _case("norm-8bit-prompt", op="norm_mx8", T=4001, d=1536),
        # the smallest configuration, three short sequences of which one is empty: launches and latency
        _case("balance-tiny", op="balance", dtype="f32", T=128, d=64, E=8, k=2, n_seq=3),
        # the fine-grained pool with its softmax router, packed ragged sequences with padding behind them, hot experts
        _case("balance-fine-grained-ragged", op="balance", T=16384, d=1024, E=512, k=8, n_seq=37, padded=True, router="softmax",
              skew="hot"),
        # serving the largest pool: four sequences decoding, and its largest batch
        _case("experts-decode-few", op="experts", T=4, d=1536, f=4096, E=192, k=2),
        _case("experts-largest", op="experts", T=32768, d=1536, f=4096, E=192, k=2),
        # a batch of sequences decoding with the fine-grained pool
        _case("experts-decode-batch-fine-grained", op="experts", T=48, d=1024, f=704, E=512, k=8),
        # odd sizes under skew: a prompt on a pool whose widths are no multiples of 128
        _case("experts-odd-pool-prompt-hot", op="experts", T=1501, d=832, f=1472, E=90, k=3, skew="hot"),
        # weights to 8 bits: the small pool's gate and up matrices, from a bfloat16 checkpoint; a float matrix of a ragged width
        _case("quantize-gate-up", op="quantize", T=64 * 4096, d=768),
        _case("quantize-f32-ragged", op="quantize", dtype="f32", T=2001, d=416),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["norm", "norm_mx8", "balance", "experts", "experts", "quantize"])
        if op == "norm":
            c = _case(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]), T=_log_int(rng, 1, 65536), residual=rng.random() < 0.8)
            c["d"] = 64 * _log_int(rng, 1, 128) if c["dtype"] == "bf16" else _log_int(rng, 1, 8192)
            ok = c["T"] * c["d"] * (1 if c["dtype"] == "bf16" else 2) <= 32768 * 1536
        elif op == "norm_mx8":
            c = _case(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]), T=_log_int(rng, 1, 32768), residual=rng.random() < 0.8)
            c["d"] = 64 * _log_int(rng, 1, 128) if c["dtype"] == "bf16" else 32 * _log_int(rng, 1, 256)
            ok = c["T"] * c["d"] * (1 if c["dtype"] == "bf16" else 2) <= 32768 * 1536
        elif op == "balance":
            c = _case(op=op, T=_log_int(rng, 1, 131072), E=rng.choice([8 * _log_int(rng, 1, 64), _log_int(rng, 1, 512)]),
                      k=rng.choice([1, 2, 2, 3, 4, 6, 8]), n_seq=_log_int(rng, 1, 256), padded=rng.random() < 0.5,
                      router=rng.choice(["norm", "softmax"]), skew=rng.choice(["none", "hot"]))
            ok = c["k"] <= c["E"] and c["T"] * c["E"] <= 32768 * 512
        elif op == "quantize":
            c = _case(op=op, dtype=rng.choice(["bf16", "f32"]), T=_log_int(rng, 1, 1 << 20), d=32 * _log_int(rng, 1, 256))
            ok = c["T"] * c["d"] <= 64 * 4096 * 768
        else:
            c = _case(op=op, T=_log_int(rng, 1, 16384), d=64 * _log_int(rng, 1, 24), f=64 * _log_int(rng, 1, 64),
                      k=rng.choice([1, 2, 2, 3, 4, 8]), skew=rng.choice(["none", "none", "hot"]))
            c["E"] = rng.choice([8 * _log_int(rng, 1, 64), _log_int(rng, 1, 500)])
            big = _case(op=op, T=32768, d=1536, f=4096, E=192, k=2)
            ok = (c["k"] <= c["E"] and c["E"] * c["d"] * c["f"] <= 192 * 1536 * 4096 and
                  work(c)["flops"] * (3 if c["skew"] == "hot" else 1) <= work(big)["flops"] and c["T"] * c["k"] * (c["d"] + c["f"]) <= 1 << 28)
        if ok:
            return c


def work(case):
    """What a pass cannot do without: inputs read once, outputs written once."""
    c = _case(**{k: v for k, v in case.items() if k != "name"})
    T, d, f, E, k = (c[n] for n in ("T", "d", "f", "E", "k"))
    act = 2 if c["dtype"] == "bf16" else 4
    res = 1 if c["residual"] else 0
    if c["op"] == "norm":          # x, residual, dy, dh in; h, y, dx and the float d_weight out
        return {"bytes": act * T * d * (6.0 + res) + act * d + 4.0 * d, "flops": 16.0 * T * d}
    if c["op"] == "norm_mx8":
        return {"bytes": act * T * d * (3.0 + res) + T * d * 33.0 / 32.0 + act * d, "flops": 8.0 * T * d}
    if c["op"] == "balance":       # logits in, their gradient out, picks in, counts out
        return {"bytes": 8.0 * T * E + 4.0 * T * k + 4.0 * c["n_seq"] * E, "flops": 12.0 * T * E}
    if c["op"] == "quantize":
        return {"bytes": T * d * (act + 33.0 / 32.0), "flops": 3.0 * T * d}
    reached = E * (1.0 - (1.0 - k / E) ** T)               # experts with rows, under even use
    return {"bytes": (3.0 * d * f * reached + T * d) * 33.0 / 32.0 + 2.0 * T * k * d, "flops": 6.0 * T * k * d * f}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _normal(shape, gen, dtype, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device=DEVICE).normal_(0.0, std, generator=gen).to(dtype)


def _to_mx8(v):
    """(8-bit values [rows, cols], scale bytes [ceil(cols / 128), rows, 4]) of a float matrix."""
    rows, cols = v.shape
    b = v.view(rows, cols // 32, 32)
    m, e = torch.frexp(b.abs().amax(dim=2))                # amax = m 2^e, 0.5 <= m < 1; 448 = 0.875 * 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-127)
    e = torch.where(m == 0, torch.full_like(e, -127), e)
    q = torch.ldexp(b, -e.unsqueeze(2)).to(torch.float8_e4m3fn).view(rows, cols)
    blocks = -(-cols // 128) * 4
    s = torch.full((rows, blocks), 127, dtype=torch.uint8, device=v.device)
    s[:, :cols // 32] = (e + 127).to(torch.uint8)
    return q, s.view(rows, blocks // 4, 4).permute(1, 0, 2).contiguous()


def _from_mx8(q, scale, dtype):
    """The values that an 8-bit matrix stands for."""
    rows, cols = q.shape
    e = scale.permute(1, 0, 2).reshape(rows, -1)[:, :cols // 32].to(torch.int32) - 127
    v = q.to(dtype).view(rows, cols // 32, 32)
    return torch.ldexp(v, e.unsqueeze(2)).view(rows, cols)


def _hot(E, rng):
    bias = np.zeros(E, dtype=np.float32)
    bias[rng.permutation(E)[: max(1, E // 5)]] = 1.5
    return torch.from_numpy(bias).to(DEVICE)


def _offsets(T, n, padded, rng):
    """Ragged sequences: every fifth one empty (where there are several), lengths spread by their logarithm."""
    w = np.exp(rng.normal(0.0, 0.7, n))
    if n > 1:
        w[rng.permutation(n)[: max(1, n // 5)]] = 0.0
    end = int(T * (0.93 if padded else 1.0))
    return np.concatenate([[0], np.round(np.cumsum(w) / w.sum() * end)]).astype(np.int32)


def prepare(case, seed):
    c = _case(**{k: v for k, v in case.items() if k != "name"})
    T, d, f, E, k = (c[n] for n in ("T", "d", "f", "E", "k"))
    act = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    s = dict(case=c)
    mx8 = lambda rows, cols: (torch.zeros((rows, cols), dtype=torch.uint8, device=DEVICE),  # noqa: E731
                              torch.zeros((-(-cols // 128), rows, 4), dtype=torch.uint8, device=DEVICE))
    if c["op"] in ("norm", "norm_mx8"):
        s["x"] = _normal((T, d), gen, act)
        s["residual"] = _normal((T, d), gen, act, 3.0) if c["residual"] else None
        s["weight"] = (1.0 + _normal((d,), gen, torch.float32, 0.1)).to(act)
        s["h"], s["y"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        if c["op"] == "norm":
            s["dy"], s["dh"] = _normal((T, d), gen, act), _normal((T, d), gen, act)
            s["dx"], s["d_weight"] = torch.empty_like(s["x"]), torch.empty(d, dtype=torch.float32, device=DEVICE)
        else:
            s["q"], s["scale"] = mx8(T, d)
    elif c["op"] == "balance":
        s["logits"] = _normal((T, E), gen, torch.float32, 2.0 if c["router"] == "softmax" else 30.0)
        if c["skew"] == "hot":
            s["logits"] += (1.0 if c["router"] == "softmax" else 15.0) * _hot(E, rng)
        s["topk_idx"] = torch.topk(s["logits"], k, dim=1).indices.to(torch.int32).contiguous()
        s["offsets"] = torch.from_numpy(_offsets(T, c["n_seq"], c["padded"], rng)).to(DEVICE)
        s["counts"] = torch.zeros((c["n_seq"], E), dtype=torch.int32, device=DEVICE)
        s["loss"], s["d_sigma"] = (torch.zeros(1, dtype=torch.float32, device=DEVICE) for _ in range(2))
        s["d_logits"] = torch.empty((T, E), dtype=torch.float32, device=DEVICE)
    elif c["op"] == "quantize":
        s["v"] = _normal((T, d), gen, act, WEIGHT_STD)
        s["q"], s["scale"] = mx8(T, d)
    else:
        S = T * k
        z = _normal((T, E), gen, torch.float32)
        if c["skew"] == "hot":
            z += _hot(E, rng)
        expert = torch.topk(z, k, dim=1).indices.reshape(-1)
        s["slot_of_row"] = torch.argsort(expert, stable=True).to(torch.int32)
        rows = torch.bincount(expert, minlength=E)
        s["offsets"] = torch.cat([rows.new_zeros(1), rows.cumsum(0)]).to(torch.int32)
        s["most_rows"] = int(rows.max())
        s["x"] = _to_mx8(_normal((T, d), gen, torch.float32))
        s["w_gate_up"] = _to_mx8(_normal((E * 2 * f, d), gen, torch.float32, WEIGHT_STD))
        s["w_down"] = _to_mx8(_normal((E * d, f), gen, torch.float32, WEIGHT_STD))
        s["h"] = mx8(S, f)
        s["y"] = torch.empty((S, d), dtype=torch.bfloat16, device=DEVICE)
    if own:
        import paper_2605_06665_amd as U
        dtype = U.F32 if c["dtype"] == "f32" else U.BF16
        if c["op"] == "balance" or c["op"] == "quantize":
            dtype = U.F32 if c["dtype"] == "f32" or d % 64 else U.BF16
        s["dtype"] = U.BF16 if c["dtype"] == "bf16" else U.F32
        s["shape"] = U.Shape(T=T, d_model=d, d_ff=f, E=E, k=k, L=1, dtype=dtype, sigma=SIGMA, c=C, eps=EPS, alpha_pool=ALPHA,
                             router=U.ROUTER_SOFTMAX if c["router"] == "softmax" else U.ROUTER_NORM)
        if c["op"] != "quantize":
            s["ws"] = torch.empty(U.workspace_bytes(s["shape"]), dtype=torch.uint8, device=DEVICE)
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def _own(s):
    import paper_2605_06665_amd as U
    c, sh = s["case"], s.get("shape")
    if c["op"] == "norm":
        U.rmsnorm(sh, s["x"], s["residual"], s["weight"], NORM_EPS, s["h"], s["y"], None, None)
        U.rmsnorm_bwd(sh, s["h"], s["weight"], s["dy"], s["dh"], NORM_EPS, s["dx"], s["d_weight"], s["ws"])
    elif c["op"] == "norm_mx8":
        U.rmsnorm(sh, s["x"], s["residual"], s["weight"], NORM_EPS, s["h"], s["y"], s["q"], s["scale"])
    elif c["op"] == "balance":
        U.seq_balance_loss(sh, c["n_seq"], s["offsets"], ALPHA, s["logits"], s["topk_idx"], s["counts"], s["loss"], s["d_logits"],
                           s["d_sigma"], s["ws"])
    elif c["op"] == "quantize":
        U.quantize_mx8(s["dtype"], c["T"], c["d"], s["v"], s["q"], s["scale"])
    else:
        U.expert_ffn_fwd_mx8(sh, *s["x"], s["slot_of_row"], s["offsets"], *s["w_gate_up"], *s["w_down"], *s["h"], s["y"], s["ws"])
    return s


def _plain_norm(s):
    """h, its reciprocal norm and y, in float."""
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    rs = torch.rsqrt((h * h).mean(dim=1, keepdim=True) + NORM_EPS)
    return h, rs, h * rs * s["weight"].float()


def _plain_balance(s):
    c, z, off = s["case"], s["logits"], s["offsets"].to(torch.int64)
    T, E, B = c["T"], c["E"], c["n_seq"]
    t = torch.arange(T, device=z.device)
    seq = (torch.searchsorted(off, t, right=True) - 1).clamp(0, B - 1)
    inside = ((t >= off[0]) & (t < off[-1]))
    flat = (seq.unsqueeze(1) * E + s["topk_idx"].to(torch.int64)).reshape(-1)
    n = torch.zeros(B * E, dtype=torch.int32, device=z.device)
    n.index_add_(0, flat, inside.to(torch.int32).repeat_interleave(c["k"]))
    n = n.view(B, E)
    length = (off[1:] - off[:-1]).float()
    used = (length > 0).sum()
    coef = ALPHA * E * n.float() / (c["k"] * length.clamp(min=1.0) * length.clamp(min=1.0) * used).unsqueeze(1)
    g = coef[seq] * inside.unsqueeze(1)
    if c["router"] == "softmax":
        p = torch.exp(z - z.amax(dim=1, keepdim=True))
        p = p / p.sum(dim=1, keepdim=True)
        gp = g * p
        dz = gp - p * gp.sum(dim=1, keepdim=True)
        loss, d_sigma = gp.sum(), torch.zeros((), device=z.device)
    else:
        norm = torch.sqrt((z * z).sum(dim=1, keepdim=True))
        inv = 1.0 / (norm + EPS)
        zh = z * inv
        loss = (g * (SIGMA * C) * zh.clamp(min=0.0)).sum()
        gz = torch.where(zh > 0, g * (SIGMA * C), torch.zeros_like(g))
        dz = gz * inv - z * ((gz * z).sum(dim=1, keepdim=True) * inv * inv / norm)
        d_sigma = loss / SIGMA
    return n, loss.reshape(1), dz, d_sigma.reshape(1)


def _plain_rows(s):
    """Row numbers [E, most rows of an expert] and which of them are the expert's."""
    off = s["offsets"].to(torch.int64)
    row = off[:-1].unsqueeze(1) + torch.arange(s["most_rows"], device=off.device)
    return row, row < off[1:].unsqueeze(1)


def _plain_experts(s):
    c = s["case"]
    d, f, E, k = (c[n] for n in ("d", "f", "E", "k"))
    row, mine = _plain_rows(s)
    token = s["slot_of_row"].to(torch.int64)[row.clamp(max=c["T"] * k - 1)] // k
    x = _from_mx8(*s["x"], torch.float32)[token.reshape(-1)].view(E, -1, d)
    w = _from_mx8(*s["w_gate_up"], torch.float32).view(E, 2 * f, d).transpose(1, 2).contiguous()
    ab = torch.bmm(x, w)
    a, b = ab[..., :f], ab[..., f:]
    h = (a / (1.0 + torch.exp(-a)) * b).reshape(-1, f)
    h = _from_mx8(*_to_mx8(h), torch.float32).view(E, -1, f)
    w = _from_mx8(*s["w_down"], torch.float32).view(E, d, f).transpose(1, 2).contiguous()
    y = torch.bmm(h, w)
    out = torch.zeros((c["T"] * k + 1, d), dtype=torch.bfloat16, device=x.device)
    out[torch.where(mine, row, torch.full_like(row, c["T"] * k)).reshape(-1)] = y.view(-1, d).to(torch.bfloat16)
    return out[:-1]


def _plain(s):
    c = s["case"]
    if c["op"] == "norm":
        h, _, y = _plain_norm(s)
        act = s["x"].dtype
        hr, dy = h.to(act).float(), s["dy"].float()            # the backward pass starts from the stored h
        rs = torch.rsqrt((hr * hr).mean(dim=1, keepdim=True) + NORM_EPS)
        g = dy * s["weight"].float()
        dx = rs * g - hr * (rs * rs * rs * (g * hr).mean(dim=1, keepdim=True)) + s["dh"].float()
        return dict(h=h.to(act), y=y.to(act), dx=dx.to(act), d_weight=(dy * hr * rs).sum(dim=0))
    if c["op"] == "norm_mx8":
        h, _, y = _plain_norm(s)
        q, scale = _to_mx8(y)
        return dict(h=h.to(s["x"].dtype), y=y.to(s["x"].dtype), q=q, scale=scale)
    if c["op"] == "balance":
        n, loss, dz, d_sigma = _plain_balance(s)
        return dict(counts=n, loss=loss, d_logits=dz, d_sigma=d_sigma)
    if c["op"] == "quantize":
        q, scale = _to_mx8(s["v"].float())
        return dict(q=q, scale=scale)
    return dict(y=_plain_experts(s))


_OUTPUTS = dict(norm=("h", "y", "dx", "d_weight"), norm_mx8=("h", "y", "q", "scale"), balance=("counts", "loss", "d_logits", "d_sigma"),
                quantize=("q", "scale"), experts=("y",))


def run(state):
    got = _own(state) if own else _plain(state)
    out = {n: got[n] for n in _OUTPUTS[state["case"]["op"]]}
    if "q" in out:                                             # the values that the bytes stand for
        out["q"], out["scale"] = out["q"].view(torch.float8_e4m3fn), out["scale"].view(torch.float8_e8m0fnu)
    return out


# ---------------------------------------------------------------------------------------------------------------
# 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------------------------
def _exact_mx8(v):
    """Values / 2^e rounded to the e4m3 grid, and 2^e in the layout of the scales."""
    rows, cols = v.shape
    b = v.reshape(rows, -1, 32)
    amax = b.abs().amax(dim=2)
    e = torch.ceil(torch.log2(torch.clamp(amax, min=1e-300) / 448.0))
    e = torch.where(amax > 448.0 * torch.exp2(e), e + 1, e)    # the logarithm's own rounding
    e = torch.where(amax <= 448.0 * torch.exp2(e - 1), e - 1, e).clamp(min=-127.0)
    u = b * torch.exp2(-e).unsqueeze(2)
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3.0)      # below 2^-6 the grid is even
    u = torch.round(u / step) * step
    blocks = -(-cols // 128) * 4
    s = torch.ones((rows, blocks), dtype=v.dtype, device=v.device)
    s[:, :cols // 32] = torch.exp2(e)
    return u.reshape(rows, cols), s.reshape(rows, -1, 4).permute(1, 0, 2).contiguous()


def _exact_values(q, scale):
    rows, cols = q.shape
    s = torch.exp2(scale.permute(1, 0, 2).reshape(rows, -1)[:, :cols // 32].double() - 127.0)
    return (q.double().reshape(rows, -1, 32) * s.unsqueeze(2)).reshape(rows, cols)


def _exact_experts(s):
    c = s["case"]
    d, f, E, k = (c[n] for n in ("d", "f", "E", "k"))
    x, off = _exact_values(*s["x"]), s["offsets"].tolist()
    y = torch.zeros((c["T"] * k, d), dtype=torch.float64, device=x.device)
    wgu = [w.reshape((E, 2 * f, -1) if i == 0 else (w.shape[0], E, 2 * f, 4)) for i, w in enumerate(s["w_gate_up"])]
    wd = [w.reshape((E, d, -1) if i == 0 else (w.shape[0], E, d, 4)) for i, w in enumerate(s["w_down"])]
    for e in range(E):
        r0, r1 = off[e], off[e + 1]
        if r0 == r1:
            continue
        xe = x[torch.div(s["slot_of_row"][r0:r1].long(), k, rounding_mode="floor")]
        ab = xe @ _exact_values(wgu[0][e], wgu[1][:, e]).T
        a, b = ab[:, :f], ab[:, f:]
        u, sc = _exact_mx8(a * torch.sigmoid(a) * b)
        hv = (u.reshape(r1 - r0, -1, 32) * sc.permute(1, 0, 2).reshape(r1 - r0, -1)[:, :f // 32].unsqueeze(2)).reshape(r1 - r0, f)
        y[r0:r1] = hv @ _exact_values(wd[0][e], wd[1][:, e]).T
    return y


def _exact_balance(s):
    """Sequence by sequence."""
    c, z, off = s["case"], s["logits"].double(), s["offsets"].tolist()
    E, k = c["E"], c["k"]
    counts = torch.zeros((c["n_seq"], E), dtype=torch.int32, device=z.device)
    dz, loss = torch.zeros_like(z), z.new_zeros(())
    used = sum(b > a for a, b in zip(off, off[1:]))
    for i, (a, b) in enumerate(zip(off, off[1:])):
        if a == b:
            continue
        counts[i] = torch.bincount(s["topk_idx"][a:b].reshape(-1).long(), minlength=E).to(torch.int32)
        zs = z[a:b].clone().requires_grad_(True)
        if c["router"] == "softmax":
            score = torch.softmax(zs, dim=1)
        else:
            score = SIGMA * C * torch.relu(zs / (zs.norm(dim=1, keepdim=True) + EPS))
        part = ALPHA / used * (E / (k * (b - a)) * counts[i].double() * score.mean(dim=0)).sum()
        dz[a:b] = torch.autograd.grad(part, zs)[0]
        loss = loss + part.detach()
    d_sigma = loss / SIGMA if c["router"] == "norm" else torch.zeros_like(loss)
    return dict(counts=counts, loss=loss.reshape(1), d_logits=dz, d_sigma=d_sigma.reshape(1))


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["op"] in ("norm", "norm_mx8"):
        w = s["weight"].double()
        h = s["x"].double() + (s["residual"].double() if s["residual"] is not None else 0.0)
        y = h / torch.sqrt(h.square().mean(dim=1, keepdim=True) + NORM_EPS) * w
        if c["op"] == "norm_mx8":
            q, scale = _exact_mx8(y)
            return dict(h=h, y=y, q=q, scale=scale)
        hs = h.to(s["x"].dtype).double().requires_grad_(True)
        wg = w.clone().requires_grad_(True)
        out = hs / torch.sqrt(hs.square().mean(dim=1, keepdim=True) + NORM_EPS) * wg
        dx, dw = torch.autograd.grad(out, (hs, wg), s["dy"].double())
        return dict(h=h, y=y, dx=dx + s["dh"].double(), d_weight=dw)
    if c["op"] == "balance":
        return _exact_balance(s)
    if c["op"] == "quantize":
        q, scale = _exact_mx8(s["v"].double())
        return dict(q=q, scale=scale)
    return dict(y=_exact_experts(s))
