"""Norm with residual, its 8-bit output and its backward pass against float64.

Tolerances: a stored value is off by half a step of its type (bfloat16 2^-8, float 2^-24 of the value).  Float arithmetic before that:
a sum is a chain of at most 16 terms per lane, 6 steps between lanes and 16 between wavefronts, each 2^-24 of sums of magnitudes, the
square root halves its share, and about six more roundings follow: C = 48 steps of 2^-24 cover it, on the magnitudes that are added."""
import numpy as np
import pytest

from oracle import sublayer_oracle as O
from tests.gpu_util import dev, host, round_act

pytestmark = pytest.mark.gpu

EPS = 1e-6
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
C = 48 * 2.0 ** -24


def lib():
    import paper_2605_06665_amd as U
    return U


def shape(T, d, dtype):
    U = lib()
    return U.Shape(T=T, d_model=d, d_ff=64, E=8, k=2, L=1, dtype=U.BF16 if dtype == "bf16" else U.F32, sigma=1.0, c=2.5, eps=1e-6,
                   alpha_pool=0.01)


def rows(T, d, dtype, seed, scale=1.0):
    return round_act(np.random.default_rng(seed).standard_normal((T, d)) * scale, dtype)


def like(t, shift=0):
    """An empty tensor of t's shape, `shift` elements past an address aligned to 256 bytes."""
    import torch
    return torch.full((t.numel() + shift,), float("nan"), dtype=t.dtype, device="cuda")[shift:].view(t.shape)


def shifted(t, shift):
    o = like(t, shift)
    o.copy_(t)
    return o


def mx8_of(T, d):
    import torch
    return (torch.full((T, d), 0x55, dtype=torch.uint8, device="cuda"),
            torch.full(lib().mx8_scale_shape(T, d), 255, dtype=torch.uint8, device="cuda"))


def act_err(got, want, dtype, slack):
    """Largest of |got - want| / what it may be."""
    want = np.asarray(want, np.float64)
    return np.max(np.abs(got.astype(np.float64) - want) / (HALF[dtype] * np.abs(want) + slack + 1e-30))


# every form of the kernels: the widths on both sides of each
CASES = [("bf16", T, d) for T, d in ((1, 64), (3, 512), (5, 576), (257, 1024), (9, 1088), (130, 1536), (66, 1600), (4, 2048), (7, 2112),
                                      (2, 4096), (5, 4160), (3, 8192), (2, 8256), (1, 16384), (3000, 128))] + \
        [("f32", T, d) for T, d in ((1, 1), (3, 5), (65, 31), (4, 252), (2, 256), (9, 257), (5, 260), (6, 512), (3, 1000), (2, 1023),
                                     (2, 1028), (5, 2048), (3, 2052), (2, 4096), (2, 4099), (3, 4100), (1, 16384), (2, 16381), (2501, 40))]


@pytest.mark.parametrize("dtype,T,d", CASES)
@pytest.mark.parametrize("residual", [True, False])
def test_forward(dtype, T, d, residual):
    import torch
    U, sh = lib(), shape(T, d, dtype)
    x, r = rows(T, d, dtype, 1), rows(T, d, dtype, 2, 3.0) if residual else None
    w = round_act(1.0 + 0.1 * np.random.default_rng(3).standard_normal(d), dtype)
    h_ref, y_ref = O.rmsnorm(x, r, w, EPS)
    gx, gr, gw = dev(x, dtype), dev(r, dtype) if residual else None, dev(w, dtype)
    h, y = like(gx), like(gx)
    q, s = mx8_of(T, d) if d % 32 == 0 else (None, None)
    U.rmsnorm(sh, gx, gr, gw, EPS, h, y, q, s)
    torch.cuda.synchronize()
    assert act_err(host(h), h_ref, dtype, 2.0 ** -24 * np.abs(h_ref)) <= 1
    assert act_err(host(y), y_ref, dtype, C * np.abs(y_ref)) <= 1
    if q is None:
        return
    sc = s.cpu().numpy()
    assert (np.transpose(sc, (1, 0, 2)).reshape(T, -1)[:, d // 32:] == 127).all()
    e = np.repeat(np.transpose(sc, (1, 0, 2)).reshape(T, -1)[:, :d // 32].astype(int) - 127, 32, axis=1)
    back = O.from_mx8(q.cpu().numpy(), sc)
    # half a step of e4m3 (2^-4 of a normal value, 2^-10 2^e below), and no scale larger than the values need
    assert (np.abs(back - y_ref) <= np.maximum(2.0 ** -4 * np.abs(y_ref), 2.0 ** (e - 10.0)) + 2 * C * np.abs(y_ref) + 1e-45).all()
    amax = np.abs(y_ref).reshape(T, -1, 32).max(axis=2).repeat(32, axis=1)
    assert (amax * (1 + C) > 448.0 * 2.0 ** (e - 1.0))[e > -127].all()
    if dtype == "f32":          # the float y is what the bytes are made from
        qr, sr = O.to_mx8(host(y))
        assert np.array_equal(sr, sc) and np.array_equal(qr, q.cpu().numpy())
    # y and h left out: the same bytes
    q2, s2 = mx8_of(T, d)
    U.rmsnorm(sh, gx, gr, gw, EPS, None, None, q2, s2)
    assert torch.equal(q, q2) and torch.equal(s, s2)


@pytest.mark.parametrize("dtype,T,d", CASES)
@pytest.mark.parametrize("with_dh", [True, False])
def test_backward(dtype, T, d, with_dh):
    import torch
    U, sh = lib(), shape(T, d, dtype)
    h, dy = rows(T, d, dtype, 4, 2.0), rows(T, d, dtype, 5)
    dh = rows(T, d, dtype, 6) if with_dh else None
    w = round_act(1.0 + 0.1 * np.random.default_rng(7).standard_normal(d), dtype)
    dx_ref, dw_ref = O.rmsnorm_bwd(h, w, dy, dh, EPS)
    ws = torch.full((U.workspace_bytes(sh),), 255, dtype=torch.uint8, device="cuda")
    args = dev(h, dtype), dev(w, dtype), dev(dy, dtype), dev(dh, dtype) if with_dh else None
    dx, dw = like(args[0]), torch.full((d,), float("nan"), device="cuda")
    U.rmsnorm_bwd(sh, *args, EPS, dx, dw, ws)
    torch.cuda.synchronize()
    s = 1.0 / np.sqrt(np.mean(h.astype(np.float64) ** 2, axis=1, keepdims=True) + EPS)
    g = np.abs(w * dy.astype(np.float64))
    mag = s * g + np.abs(h) * s ** 3 * np.mean(g * np.abs(h), axis=1, keepdims=True) + (np.abs(dh) if with_dh else 0.0)
    assert act_err(host(dx), dx_ref, dtype, C * mag) <= 1
    # a column's sum: the rows of a wavefront one after the other (at most T / 4 of them, less in many workgroups), then the partial sums
    terms = np.sum(np.abs(dy.astype(np.float64) * h * s), axis=0)
    assert (np.abs(host(dw) - dw_ref) <= (C + (min(T, 64) + T / 512.0) * 2.0 ** -24) * terms + 1e-30).all()
    # dx in the place of dy and of dh
    for inplace in (2, 3) if with_dh else (2,):
        a = list(dev(t, dtype) if t is not None else None for t in (h, w, dy, dh))
        dw2 = torch.zeros_like(dw)
        U.rmsnorm_bwd(sh, *a, EPS, a[inplace], dw2, ws)
        assert torch.equal(a[inplace], dx) and torch.equal(dw, dw2)


@pytest.mark.parametrize("dtype,T,d", [("bf16", 5, 192), ("bf16", 3, 1088), ("bf16", 2, 4160), ("f32", 7, 96), ("f32", 3, 1024), ("f32", 2, 4128)])
def test_any_address(dtype, T, d):
    """Tensors one element past a 16-byte address: single loads, and the values of the wide ones up to the order of the sums."""
    import torch
    U, sh = lib(), shape(T, d, dtype)
    gx, gr, gw = dev(rows(T, d, dtype, 1), dtype), dev(rows(T, d, dtype, 2), dtype), dev(rows(1, d, dtype, 3)[0], dtype)
    h, y, (q, s) = like(gx), like(gx), mx8_of(T, d)
    U.rmsnorm(sh, gx, gr, gw, EPS, h, y, q, s)
    h1, y1 = like(gx, 1), like(gx, 1)
    q1, s1 = torch.zeros(T * d + 1, dtype=torch.uint8, device="cuda")[1:].view(T, d), torch.zeros(s.numel() + 1, dtype=torch.uint8, device="cuda")[1:].view(s.shape)
    U.rmsnorm(sh, shifted(gx, 1), shifted(gr, 1), shifted(gw, 1), EPS, h1, y1, q1, s1)
    assert torch.equal(h, h1)
    assert np.all(np.abs(host(y1).astype(np.float64) - host(y)) <= (2 * HALF[dtype] + 2 * C) * np.abs(host(y)))
    a, b = O.from_mx8(q.cpu().numpy(), s.cpu().numpy()), O.from_mx8(q1.cpu().numpy(), s1.cpu().numpy())
    assert np.mean(a != b) < 1e-2 and np.all(np.abs(a - b) <= 2.0 ** -3 * np.abs(a) + 1e-6)
    ws = torch.empty(U.workspace_bytes(sh), dtype=torch.uint8, device="cuda")
    dy, dh = gx, gr
    dx, dw, dx1, dw1 = like(gx), like(gw.float()), like(gx, 1), like(gw.float(), 1)
    U.rmsnorm_bwd(sh, h, gw, dy, dh, EPS, dx, dw, ws)
    U.rmsnorm_bwd(sh, shifted(h, 1), shifted(gw, 1), shifted(dy, 1), shifted(dh, 1), EPS, dx1, dw1, ws)
    dx_ref, dw_ref = O.rmsnorm_bwd(host(h), host(gw), host(dy), host(dh), EPS)
    hs = host(h).astype(np.float64)
    sc = 1.0 / np.sqrt(np.mean(hs ** 2, axis=1, keepdims=True) + EPS)
    g = np.abs(host(gw) * host(dy).astype(np.float64))
    mag = sc * g + np.abs(hs) * sc ** 3 * np.mean(g * np.abs(hs), axis=1, keepdims=True) + np.abs(host(dh))
    assert act_err(host(dx1), dx_ref, dtype, C * mag) <= 1
    assert np.all(np.abs(host(dw1) - dw_ref) <= C * np.sum(np.abs(host(dy) * hs * sc), axis=0) + 1e-30)


def test_in_place_residual_and_rows_that_are_zero_or_not_finite():
    import torch
    U, T, d = lib(), 6, 128
    sh = shape(T, d, "bf16")
    x = rows(T, d, "bf16", 8)
    x[1] = 0.0
    x[3, 40] = np.inf
    x[4, 70] = np.nan
    gx, gw = dev(x, "bf16"), dev(np.ones(d, np.float32), "bf16")
    r = torch.zeros_like(gx)
    y, (q, s) = like(gx), mx8_of(T, d)
    U.rmsnorm(sh, gx, r, gw, EPS, r, y, q, s)               # h is the residual itself
    torch.cuda.synchronize()
    assert torch.equal(r.view(torch.int16), (gx + 0.0).view(torch.int16)) or torch.equal(torch.nan_to_num(r), torch.nan_to_num(gx))
    _, y_ref = O.rmsnorm(x[[0, 1, 2, 5]], None, np.ones(d), EPS)
    assert act_err(host(y)[[0, 1, 2, 5]], y_ref, "bf16", C * np.abs(y_ref)) <= 1
    back = O.from_mx8(q.cpu().numpy(), s.cpu().numpy())
    assert np.isfinite(back[[0, 1, 2, 5]]).all() and (back[1] == 0).all()
    assert np.isnan(host(y)[4]).all() and np.isnan(back[4]).all()
    assert np.isnan(host(y)[3, 40]) and np.isnan(back[3, 32:64]).all()


def test_recorded_and_replayed_on_another_stream():
    import torch
    U, T, d = lib(), 300, 640
    sh = shape(T, d, "bf16")
    gx, gr, gw, dy = (dev(rows(*n, "bf16", i), "bf16") for i, n in enumerate(((T, d), (T, d), (1, d), (T, d))))
    gw = gw[0].contiguous()
    h, y, (q, s), dx, dw = like(gx), like(gx), mx8_of(T, d), like(gx), torch.zeros(d, device="cuda")
    ws = torch.empty(U.workspace_bytes(sh), dtype=torch.uint8, device="cuda")

    def run():
        U.rmsnorm(sh, gx, gr, gw, EPS, h, y, q, s)
        U.rmsnorm_bwd(sh, h, gw, dy, gr, EPS, dx, dw, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for rep in range(3):
        gx.copy_(torch.roll(gx, rep, 0))
        run()
        torch.cuda.synchronize()
        want = [t.clone() for t in (h, y, q, s, dx, dw)]
        for t in (h, y, dx, dw):
            t.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((h, y, q, s, dx, dw), want))


@pytest.mark.parametrize("dtype,T,d", [("bf16", 9, 192), ("bf16", 3, 4160), ("f32", 9, 96), ("f32", 3, 33)])
def test_backward_of_tiny_rows_without_eps(dtype, T, d):
    """s is 1e15 here: s^3 is beyond the largest float, the gradient is not."""
    import torch
    U, sh = lib(), shape(T, d, dtype)
    h, dy = rows(T, d, dtype, 21, 1e-15), rows(T, d, dtype, 22)
    w = round_act(1.0 + 0.1 * np.random.default_rng(23).standard_normal(d), dtype)
    dx_ref, dw_ref = O.rmsnorm_bwd(h, w, dy, None, 0.0)
    ws = torch.full((U.workspace_bytes(sh),), 255, dtype=torch.uint8, device="cuda")
    dx, dw = like(dev(h, dtype)), torch.full((d,), float("nan"), device="cuda")
    U.rmsnorm_bwd(sh, dev(h, dtype), dev(w, dtype), dev(dy, dtype), None, 0.0, dx, dw, ws)
    s = 1.0 / np.sqrt(np.mean(h.astype(np.float64) ** 2, axis=1, keepdims=True))
    g = np.abs(w * dy.astype(np.float64))
    mag = s * g + np.abs(h) * s ** 3 * np.mean(g * np.abs(h), axis=1, keepdims=True)
    assert act_err(host(dx), dx_ref, dtype, C * mag) <= 1
    assert (np.abs(host(dw) - dw_ref) <= 2 * C * np.sum(np.abs(dy.astype(np.float64) * h * s), axis=0)).all()


def test_more_rows_than_a_launch_takes():
    """2^21 rows go in one launch; every row is a call of its own as far as its bits go."""
    import torch
    U, d = lib(), 32
    T = 2 * (1 << 21) + 5
    x = torch.randn(T, d, device="cuda")
    w = torch.randn(d, device="cuda")
    y, (q, s) = like(x), mx8_of(T, d)
    U.rmsnorm(shape(T, d, "f32"), x, None, w, EPS, None, y, q, s)
    for lo, hi in ((0, 1 << 20), (1 << 20, (1 << 21) + 7), ((1 << 21) + 7, 1 << 22), ((1 << 22) - 3, T)):
        n = hi - lo
        y2, (q2, s2) = like(x[lo:hi]), mx8_of(n, d)
        U.rmsnorm(shape(n, d, "f32"), x[lo:hi].clone(), None, w, EPS, None, y2, q2, s2)
        assert torch.equal(y2, y[lo:hi]) and torch.equal(q2, q[lo:hi]) and torch.equal(s2, s[:, lo:hi])


def test_backward_of_the_most_rows():
    """Next to 2^31 rows of one value: the last ones as a call of their own, the weight's gradient against 64 bits."""
    import torch
    U, T, n = lib(), (1 << 31) - 5, 1000
    sh = U.Shape(T=T, d_model=1, d_ff=64, E=1, k=1, L=1, dtype=U.F32, sigma=1.0, c=2.5, eps=1e-6, alpha_pool=0.01)
    h, dy = torch.randn((T, 1), device="cuda"), torch.randn((T, 1), device="cuda")
    w = torch.full((1,), 1.25, device="cuda")
    dx, dw = torch.empty_like(h), torch.full((1,), float("nan"), device="cuda")
    U.rmsnorm_bwd(sh, h, w, dy, None, 0.5, dx, dw, torch.empty(U.workspace_bytes(sh), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    sh2, dx2 = shape(n, 1, "f32"), torch.empty((n, 1), device="cuda")
    U.rmsnorm_bwd(sh2, h[-n:].clone(), w, dy[-n:].clone(), None, 0.5, dx2, torch.empty_like(dw), torch.empty(U.workspace_bytes(sh2), dtype=torch.uint8, device="cuda"))
    assert torch.equal(dx[-n:], dx2)
    want = terms = 0.0
    for a, b in zip(h.split(1 << 28), dy.split(1 << 28)):
        t = a.double()
        t = b.double() * t / torch.sqrt(t * t + 0.5)
        want, terms = want + float(t.sum()), terms + float(t.abs().sum())
    # T / 4096 rows of a wavefront one after the other, then eight wavefronts and 512 workgroups
    assert abs(float(dw) - want) <= (T / 4096.0 + 100) * 2.0 ** -24 * terms


# rows of one, four and sixteen wavefronts, in chunks of 16 bytes and value by value
@pytest.mark.parametrize("dtype,T,d", [("bf16", 9, 512), ("bf16", 7, 1536), ("bf16", 5, 4096), ("bf16", 3, 8192), ("bf16", 3, 16384), ("f32", 9, 252),
                                       ("f32", 7, 1024), ("f32", 5, 2048), ("f32", 3, 16384), ("f32", 9, 31), ("f32", 5, 1023), ("f32", 3, 4099), ("f32", 2, 16381)])
def test_outputs_in_the_place_of_inputs(dtype, T, d):
    import torch
    U, sh = lib(), shape(T, d, dtype)
    x, r, w = (dev(rows(*n, dtype, i), dtype) for i, n in enumerate(((T, d), (T, d), (1, d))))
    w = w[0].contiguous()
    h, y = like(x), like(x)
    U.rmsnorm(sh, x, r, w, EPS, h, y, None, None)
    alone = like(x)
    U.rmsnorm(sh, x, None, w, EPS, None, alone, None, None)
    for y_at in (0, 1):
        for h_at in (None, 1 - y_at):
            a = [x.clone(), r.clone()]
            U.rmsnorm(sh, *a, w, EPS, None if h_at is None else a[h_at], a[y_at], None, None)
            assert torch.equal(a[y_at], y) and torch.equal(a[1 - y_at], h if h_at is not None else (x, r)[1 - y_at])
    a = x.clone()
    U.rmsnorm(sh, a, None, w, EPS, None, a, None, None)
    assert torch.equal(a, alone)
