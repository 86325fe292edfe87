"""8-bit layout and the experts on it against float64.

Tolerances: the layout is a definition, bit for bit.  Products of e4m3 values: inside one matrix instruction a term is kept to 2^-13 of
the largest of its (at most 8) neighbours, half of that after rounding, so a sum is off by at most 8 / 2 * 2^-13 = 2^-11 of the sum of
magnitudes; H is rounded to e4m3 (half a step: 2^-4 of a normal value, 2^-10 2^e below), Y to bfloat16 (2^-8).  Element by
element that is loose, so the 2-norm is held too: float sums of random terms are off by about 1.5e-5 of the result, Y by its rounding."""
import numpy as np
import pytest

from oracle import sublayer_oracle as O
from oracle import unipool_oracle as P
from tests.gpu_util import dev, host, round_act

pytestmark = pytest.mark.gpu

ACC = 2.0 ** -11


def lib():
    import paper_2605_06665_amd as U
    return U


def new_mx8(rows, cols, fill=0x55):
    import torch
    return (torch.full((rows, cols), fill, dtype=torch.uint8, device="cuda"),
            torch.full(lib().mx8_scale_shape(rows, cols), 255, dtype=torch.uint8, device="cuda"))


def quantize(v, dtype="f32"):
    U = lib()
    q, s = new_mx8(*v.shape)
    U.quantize_mx8(U.BF16 if dtype == "bf16" else U.F32, *v.shape, dev(v, dtype), q, s)
    return q, s


def values(q, s):
    return O.from_mx8(q.cpu().numpy(), s.cpu().numpy())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 64), (63, 96), (64, 128), (65, 160), (130, 416), (1, 4096), (257, 1568), (1000, 32)])
def test_layout_bit_for_bit(dtype, rows, cols):
    g = np.random.default_rng(rows + cols)
    v = round_act(g.standard_normal((rows, cols)) * np.exp(4 * g.standard_normal((rows, 1))), dtype)
    v[0, 0] = 0.0
    v[0, 1] = -0.0
    q, s = quantize(v, dtype)
    qr, sr = O.to_mx8(v)
    assert np.array_equal(s.cpu().numpy(), sr) and np.array_equal(q.cpu().numpy(), qr)


def test_layout_of_borders_and_values_that_are_not_finite():
    """Largest values on and next to 448 times a power of two, ties between e4m3 neighbours, the smallest and largest floats."""
    rows = []
    for top in (448.0, np.nextafter(np.float32(448), np.float32(1e9)), 447.99, 449.0, 464.0, 896.0, 1.75, 1.7500001, 3.0e38, 1e-38, 1e-45, 2.6e-36, 2.7e-36, 0.0,
                np.inf, -np.inf, np.nan):
        r = np.zeros(32, np.float32)
        r[:] = np.float32(top) * np.linspace(-1, 1, 32).astype(np.float32) if np.isfinite(top) else 1.0
        r[7] = top
        rows.append(r)
    ties = np.zeros(32, np.float32)
    ties[:16] = [448, 1.0625, 1.1875, 1.3125, -1.0625, 2.0 ** -10, 3 * 2.0 ** -10, 5 * 2.0 ** -10, 2.0 ** -11, 17.0, 19.0, 21.0, 432.0, 416.0, 400.0, -424.0]
    rows.append(ties)
    v = np.stack(rows).astype(np.float32)
    q, s = quantize(v)
    qr, sr = O.to_mx8(v)
    assert np.array_equal(s.cpu().numpy(), sr) and np.array_equal(q.cpu().numpy(), qr)


def test_layout_at_any_address():
    import torch
    U = lib()
    v = np.random.default_rng(5).standard_normal((70, 96)).astype(np.float32)
    qr, sr = O.to_mx8(v)
    src = torch.empty(70 * 96 + 1, device="cuda")[1:].view(70, 96)
    src.copy_(torch.from_numpy(v))
    q = torch.zeros(70 * 96 + 1, dtype=torch.uint8, device="cuda")[1:].view(70, 96)
    s = torch.zeros(sr.size + 1, dtype=torch.uint8, device="cuda")[1:].view(sr.shape)
    U.quantize_mx8(U.F32, 70, 96, src, q, s)
    assert np.array_equal(q.cpu().numpy(), qr) and np.array_equal(s.cpu().numpy(), sr)


def routing(T, E, k, seed, skew):
    g = np.random.default_rng(seed)
    z = g.standard_normal((T, E))
    if skew == "hot":
        z[:, g.permutation(E)[:max(1, E // 5)]] += 2.0
    elif skew == "empty":                                  # most experts have no rows
        z[:, max(k, E // 4):] -= 100.0
    idx = P.topk_select(z, k)
    return P.permutation(idx, E)


def case(T, E, d, f, k, skew, seed=1):
    g = np.random.default_rng(seed)
    x = g.standard_normal((T, d)).astype(np.float32)
    wgu = (g.standard_normal((E * 2 * f, d)) * 0.05).astype(np.float32)
    wd = (g.standard_normal((E * d, f)) * 0.05).astype(np.float32)
    return [quantize(a) for a in (x, wgu, wd)]


def run(T, E, d, f, k, qs, off, sor, gathered=True):
    import torch
    U = lib()
    sh = U.Shape(T=T, d_model=d, d_ff=f, E=E, k=k, L=1, dtype=U.BF16, sigma=1.0, c=2.5, eps=1e-6, alpha_pool=0.01)
    ws = torch.full((U.workspace_bytes(sh),), 255, dtype=torch.uint8, device="cuda")
    S = T * k
    (xq, xs), wgu, wd = qs
    h, y = new_mx8(S, f), torch.full((S, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    if gathered:
        rows = (xq, xs, dev(sor.astype(np.int32)))
    else:
        tok = torch.from_numpy(sor.astype(np.int64) // k).cuda()
        rows = (xq[tok].contiguous(), xs[:, tok].contiguous(), None)
    U.expert_ffn_fwd_mx8(sh, *rows, dev(off.astype(np.int32)), *wgu, *wd, *h, y, ws)
    torch.cuda.synchronize()
    return h, y


SIZES = [
    (1, 1, 64, 64, 1, "none"), (1, 8, 128, 192, 2, "none"), (4, 6, 192, 64, 3, "none"), (16, 5, 256, 320, 2, "hot"), (17, 3, 320, 128, 1, "none"),
    (40, 4, 128, 448, 2, "none"), (64, 16, 512, 256, 2, "none"), (65, 12, 576, 704, 8, "hot"), (130, 3, 128, 128, 1, "none"), (200, 2, 192, 320, 2, "hot"),
    (300, 40, 832, 192, 3, "empty"), (500, 1, 64, 128, 1, "none"), (700, 2, 1088, 64, 1, "none"), (1000, 9, 128, 1472, 2, "hot"),
    (63, 512, 64, 64, 8, "none"), (1500, 5, 256, 256, 4, "none"),
]


# every form: weights streamed to registers, and the tiles (rows and weight rows)
FORMS = {0: [SIZES[0], SIZES[3], SIZES[6]], 64128: [SIZES[5], SIZES[7], SIZES[8], SIZES[14]], 96128: [SIZES[9], SIZES[11], SIZES[15]],
         128256: [(1600, 16, 64, 8192, 1, "none")], 192256: [(3300, 16, 64, 4160, 1, "none"), (3300, 16, 192, 4160, 1, "hot")]}


@pytest.mark.parametrize("form", FORMS)
def test_sizes_take_every_form(form):
    U = lib()
    for T, E, d, f, k, _ in FORMS[form]:
        assert U.mx8_form(U.Shape(T=T, d_model=d, d_ff=f, E=E, k=k, L=1, dtype=U.BF16, sigma=1.0, c=2.5, eps=1e-6, alpha_pool=0.01)) == form


@pytest.mark.parametrize("T,E,d,f,k,skew", SIZES + FORMS[128256] + FORMS[192256])
def test_experts(T, E, d, f, k, skew):
    import torch
    off, ros, sor = routing(T, E, k, T + E, skew)
    qs = case(T, E, d, f, k, skew)
    x, wgu, wd = (values(*q) for q in qs)
    xr, wgu, wd = x[sor // k], wgu.reshape(E, 2 * f, d), wd.reshape(E, d, f)
    (hq, hs), y = run(T, E, d, f, k, qs, off, sor)
    # H against the formula on the 8-bit operands
    h_ref = O.expert_h(xr, off, wgu)
    sc = np.transpose(hs.cpu().numpy(), (1, 0, 2)).reshape(T * k, -1)[:, :f // 32].astype(int)
    e = np.repeat(sc - 127, 32, axis=1)
    h = values(hq, hs)
    mag = np.zeros_like(h_ref)                             # what the float sums in front of H may be off by
    for ex in range(E):
        r = slice(off[ex], off[ex + 1])
        m = np.abs(xr[r]) @ np.abs(wgu[ex]).T
        ab = xr[r] @ wgu[ex].T
        a, b = ab[:, :f], ab[:, f:]
        sg = 1 / (1 + np.exp(-a))
        mag[r] = ACC * (m[:, :f] * np.abs(b) * (sg * (1 + np.abs(a) * (1 - sg))) + m[:, f:] * np.abs(a) * sg) + 1e-6 * np.abs(h_ref[r])
    assert (np.abs(h - h_ref) <= np.maximum(2.0 ** -4 * (np.abs(h_ref) + mag), 2.0 ** (e - 10.0)) + mag).all()
    amax = np.abs(h_ref).reshape(T * k, -1, 32).max(axis=2).repeat(32, axis=1)
    assert (amax + mag.reshape(T * k, -1, 32).max(axis=2).repeat(32, axis=1) > 448.0 * 2.0 ** (e - 1.0))[e > -127].all()
    # against H rounded from 64 bits: all but the values next to a border agree
    exact = O.from_mx8(*O.to_mx8(h_ref))
    assert np.linalg.norm(h - exact) <= 4e-3 * np.linalg.norm(exact)
    # Y against the formula on the kernel's own H
    y_ref = O.expert_y(h, off, wd)
    ym = np.zeros_like(y_ref)
    for ex in range(E):
        r = slice(off[ex], off[ex + 1])
        ym[r] = np.abs(h[r]) @ np.abs(wd[ex]).T
    got = host(y).astype(np.float64)
    assert (np.abs(got - y_ref) <= 2.0 ** -8 * np.abs(y_ref) + (1 + 2.0 ** -8) * ACC * ym).all()
    assert np.linalg.norm(got - y_ref) <= 2.5e-3 * np.linalg.norm(y_ref)
    # rows in group order instead of the tokens: the same bits
    (hq2, hs2), y2 = run(T, E, d, f, k, qs, off, sor, gathered=False)
    n = T * k
    assert torch.equal(hq, hq2) and torch.equal(hs.view(-1, n, 4), hs2.view(-1, n, 4)) and torch.equal(y, y2)


@pytest.mark.parametrize("T", [3, 200])
def test_rows_that_are_not_finite_stay_by_themselves(T):
    E, d, f, k = 4, 192, 128, 2
    off, ros, sor = routing(T, E, k, 3, "none")
    qs = case(T, E, d, f, k, "none")
    _, y0 = run(T, E, d, f, k, qs, off, sor)
    qs[0][1][0, 1, 2] = 255                                # token 1: the scale of its third block is NaN
    _, y1 = run(T, E, d, f, k, qs, off, sor)
    bad = sor // k == 1
    assert np.isnan(host(y1)[bad]).all() and np.array_equal(host(y1)[~bad], host(y0)[~bad])


def test_scale_bytes_past_the_columns_do_not_matter():
    """K = 192 and 64: the last words of scales are half used; bytes past the columns are not read as scales."""
    T, E, d, f, k = 150, 3, 192, 64, 2
    off, ros, sor = routing(T, E, k, 4, "none")
    qs = case(T, E, d, f, k, "none")
    (h0, _), y0 = run(T, E, d, f, k, qs, off, sor)
    for q, s in qs[:2]:
        s[1, :, 2:] = 255
    qs[2][1][0, :, 2:] = 255
    (h1, _), y1 = run(T, E, d, f, k, qs, off, sor)
    assert np.array_equal(h0.cpu().numpy(), h1.cpu().numpy()) and np.array_equal(host(y0), host(y1))


def test_recorded_and_replayed():
    import torch
    U, T, E, d, f, k = lib(), 90, 6, 256, 192, 2
    off, ros, sor = routing(T, E, k, 5, "none")
    qs = case(T, E, d, f, k, "none")
    sh = U.Shape(T=T, d_model=d, d_ff=f, E=E, k=k, L=1, dtype=U.BF16, sigma=1.0, c=2.5, eps=1e-6, alpha_pool=0.01)
    ws = torch.empty(U.workspace_bytes(sh), dtype=torch.uint8, device="cuda")
    h, y = new_mx8(T * k, f), torch.zeros((T * k, d), dtype=torch.bfloat16, device="cuda")
    g_off, g_sor, x = dev(off.astype(np.int32)), dev(sor.astype(np.int32)), torch.randn(T, d, device="cuda")

    def step():
        U.quantize_mx8(U.F32, T, d, x, *qs[0])
        U.expert_ffn_fwd_mx8(sh, *qs[0], g_sor, g_off, *qs[1], *qs[2], *h, y, ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(3):
        x.copy_(torch.roll(x, rep, 0) * 1.5)
        step()
        torch.cuda.synchronize()
        want = y.clone()
        y.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


@pytest.mark.parametrize("d,f,expected", [(64, 8192, [0, 64128, 64128, 128256, 192256, 192256]), (320, 8256, [64128, 64128, 64256, 128256, 192256, 192256])])
def test_forms_agree_bit_for_bit(d, f, expected):
    """A token's rows do not depend on how many tokens share the call, nor on the form that many take: the same first tokens in calls of
    growing size, with gathered rows whose numbers pass through LDS (several stages) and without."""
    import torch
    U, E, k = lib(), 64, 2
    T_all = 9000
    off, ros, sor = routing(T_all, E, k, 6, "none")
    g = torch.Generator(device="cuda").manual_seed(3)
    qs = []
    for rows, cols, std in ((T_all, d, 1.0), (E * 2 * f, d, 0.05), (E * d, f, 0.05)):
        v = torch.randn((rows, cols), generator=g, device="cuda") * std
        q = new_mx8(rows, cols)
        U.quantize_mx8(U.F32, rows, cols, v, *q)
        qs.append(q)
    idx = np.empty((T_all, k), np.int64)                     # the experts of every token, from the permutation
    idx.reshape(-1)[sor] = np.repeat(np.arange(E), np.diff(off))
    first, forms = None, []
    for T in (1, 3, 700, 2400, 3600, T_all):
        o, r, s = P.permutation(idx[:T], E)
        xq = (qs[0][0][:T].contiguous(), qs[0][1][:, :T].contiguous())
        forms.append(U.mx8_form(U.Shape(T=T, d_model=d, d_ff=f, E=E, k=k, L=1, dtype=U.BF16, sigma=1.0, c=2.5, eps=1e-6, alpha_pool=0.01)))
        _, y = run(T, E, d, f, k, [xq, *qs[1:]], o, s)
        mine = y[torch.from_numpy(r[:1].reshape(-1).astype(np.int64)).cuda()]
        first = mine if first is None else first
        assert torch.equal(mine, first), (T, forms[-1])
    assert forms == expected


@pytest.mark.parametrize("T,E,d,f,k", [(4, 6, 64, 192, 2), (1, 1, 64, 64, 1), (200, 5, 128, 320, 2), (130, 3, 64, 448, 1)])
def test_scale_bytes_past_the_columns_of_h(T, E, d, f, k):
    off, ros, sor = routing(T, E, k, 3, "none")
    (_, hs), _ = run(T, E, d, f, k, case(T, E, d, f, k, "none"), off, sor)
    last = hs[-1].cpu().numpy()
    assert (last[:, f % 128 // 32:] == 127).all() and (last[:, :f % 128 // 32] != 255).all()


@pytest.mark.parametrize("T", [5, 300])
def test_rows_outside_the_offsets_are_left_alone(T):
    import torch
    E, d, f, k = 4, 128, 192, 2
    off, ros, sor = routing(T, E, k, 4, "none")
    qs = case(T, E, d, f, k, "none")
    (hq, hs), y = run(T, E, d, f, k, qs, off, sor, gathered=False)
    lo, hi = int(off[1]), int(off[3])                      # the first and the last expert get none of their rows
    cut = np.clip(off, lo, hi)
    (hq2, hs2), y2 = run(T, E, d, f, k, qs, cut, sor, gathered=False)
    assert torch.equal(hq2[lo:hi], hq[lo:hi]) and torch.equal(hs2[:, lo:hi], hs[:, lo:hi]) and torch.equal(y2[lo:hi], y[lo:hi])
    for r in (slice(0, lo), slice(hi, None)):
        assert (hq2[r] == 0x55).all() and (hs2[:, r] == 255).all() and torch.isnan(y2[r]).all()


@pytest.mark.parametrize("E", [16, 2])
def test_many_gathered_rows(E):
    """Enough of them that their scales are brought into group order first (16 experts), and the same where the workspace has no room for
    that (2): the bits are those of rows in group order."""
    import torch
    U, (T, d, f, k) = lib(), (32768, 192, 8192, 2)
    g = torch.Generator(device="cuda").manual_seed(E)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    new = lambda r, c: (torch.empty((r, c), dtype=torch.uint8, device="cuda"), torch.empty(U.mx8_scale_shape(r, c), dtype=torch.uint8, device="cuda"))  # noqa: E731
    x, wgu, wd = new(T, d), new(E * 2 * f, d), new(E * d, f)
    U.quantize_mx8(U.F32, T, d, rnd(T, d) * torch.exp2(torch.randint(-20, 20, (T, 1), device="cuda", generator=g)), *x)
    U.quantize_mx8(U.F32, E * 2 * f, d, rnd(E * 2 * f, d) * 0.05, *wgu)
    U.quantize_mx8(U.F32, E * d, f, rnd(E * d, f) * 0.05, *wd)
    expert = torch.stack([torch.randperm(E, device="cuda", generator=g)[:k] if E > k else torch.arange(E, device="cuda") for _ in range(64)])
    expert = expert.repeat(T // 64, 1).flatten()
    slots = torch.argsort(expert, stable=True)
    off = torch.searchsorted(expert[slots], torch.arange(E + 1, device="cuda")).int()
    sh = U.Shape(T=T, d_model=d, d_ff=f, E=E, k=k, L=1, dtype=U.BF16, sigma=1.0, c=2.5, eps=1e-6, alpha_pool=0.01)
    ws = torch.full((U.workspace_bytes(sh),), 255, dtype=torch.uint8, device="cuda")
    tok = slots // k
    out = []
    for rows in ((x[0], x[1], slots.int()), (x[0][tok].contiguous(), x[1][:, tok].contiguous(), None)):
        h, y = new(T * k, f), torch.full((T * k, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        U.expert_ffn_fwd_mx8(sh, *rows, off, *wgu, *wd, *h, y, ws)
        out.append((*h, y))
    for a, b in zip(*out):
        assert torch.equal(a, b)
    assert torch.isfinite(out[0][2]).all()
