"""Balance loss over sequences, its gradient, and the router's backward pass that takes it in, against float64.

Tolerances: a term goes through about twenty roundings of 2^-24 (norm or exponentials, coefficient, products; exp itself 2 steps), sums
between lanes are 6 steps, the loss adds up to T / 16 partial sums 64 at a time: C = 64 steps of 2^-24 on the magnitudes that are added."""
import numpy as np
import pytest

from oracle import sublayer_oracle as O
from tests.gpu_util import dev, host

pytestmark = pytest.mark.gpu

C = 64 * 2.0 ** -24
SIGMA, CC, EPS, ALPHA = 1.2, 1.7, 1e-6, 0.3


def lib():
    import paper_2605_06665_amd as U
    return U


def shape(T, E, k, router, d=64):
    U = lib()
    return U.Shape(T=T, d_model=d, d_ff=64, E=E, k=k, L=1, dtype=U.F32, sigma=SIGMA, c=CC, eps=EPS, alpha_pool=0.01,
                   router=U.ROUTER_SOFTMAX if router == "softmax" else U.ROUTER_NORM)


def picks(z, k):
    return np.argsort(-z, axis=1, kind="stable")[:, :k].astype(np.int32)


def run(T, E, k, router, z, idx, off, grad=True, shift=0):
    import torch
    U, sh, B = lib(), shape(T, E, k, router), len(off) - 1
    ws = torch.full((U.workspace_bytes(sh),), 255, dtype=torch.uint8, device="cuda")
    gz = torch.empty(T * E + shift, device="cuda")[shift:].view(T, E)
    gz.copy_(torch.from_numpy(z))
    counts, loss = torch.full((B, E), -1, dtype=torch.int32, device="cuda"), torch.full((1,), float("nan"), device="cuda")
    dz = torch.full((T * E + shift,), float("nan"), device="cuda")[shift:].view(T, E) if grad else None
    ds = torch.full((1,), float("nan"), device="cuda") if grad else None
    U.seq_balance_loss(sh, B, dev(np.asarray(off, np.int32)), ALPHA, gz, dev(idx), counts, loss, dz, ds, ws)
    torch.cuda.synchronize()
    return counts, loss, dz, ds


def check(T, E, k, router, z, off, got):
    counts, loss, dz, ds = (host(t) for t in got)
    off = np.maximum.accumulate(np.clip(off, 0, T))
    c_ref, l_ref, dz_ref, ds_ref = O.seq_balance_loss(z, picks(z, k), off, ALPHA, router, SIGMA, CC, EPS)
    assert np.array_equal(counts, c_ref)
    assert abs(loss[0] - l_ref) <= C * abs(l_ref) + 1e-30              # its terms are all positive
    assert abs(ds[0] - ds_ref) <= C * abs(ds_ref) + 1e-30
    # a gradient is the difference of two terms of at most the larger coefficient of its sequence
    used = max(1, int((np.diff(off) > 0).sum()))
    mag = np.zeros((T, 1))
    zz = z.astype(np.float64)
    for b in range(len(off) - 1):
        n = off[b + 1] - off[b]
        if n > 0:
            coef = ALPHA * E * c_ref[b] / (k * n * used * n)
            r = slice(off[b], off[b + 1])
            if router == "softmax":
                p = np.exp(zz[r] - zz[r].max(axis=1, keepdims=True))
                p /= p.sum(axis=1, keepdims=True)
                mag[r] = (p * (coef + p @ coef[:, None])).max(axis=1, keepdims=True)
            else:
                nn = np.linalg.norm(zz[r], axis=1, keepdims=True)
                gz = np.where(zz[r] > 0, coef * SIGMA * CC, 0.0) / (nn + EPS)
                mag[r] = (gz + np.abs(zz[r]) / np.maximum(nn, 1e-30) ** 2 * (gz * np.abs(zz[r])).sum(axis=1, keepdims=True)).max(axis=1, keepdims=True)
    assert (np.abs(dz - dz_ref) <= C * mag + 1e-30).all()
    return dz


# lane layouts (4, 8, 16 logits a lane, half a row or a row of lanes), pools that are no multiple of 4, one to many sequences
SIZES = [(1, 1, 1), (5, 3, 2), (64, 4, 1), (97, 8, 2), (130, 64, 8), (33, 65, 3), (70, 96, 2), (31, 128, 8), (40, 130, 4), (50, 192, 2),
         (17, 255, 8), (90, 256, 1), (21, 260, 2), (35, 509, 8), (48, 512, 8), (2500, 12, 2), (1100, 513 - 1, 8)]


@pytest.mark.parametrize("router", ["norm", "softmax"])
@pytest.mark.parametrize("T,E,k", SIZES)
def test_loss_counts_and_gradients(T, E, k, router):
    z = np.random.default_rng(T + E).standard_normal((T, E)).astype(np.float32) * 2
    for off in ([0, T], [0, 0, T // 3, T // 3, T], [T // 4, T // 2, T - T // 5], list(range(0, T + 1, max(1, T // 37)))):
        check(T, E, k, router, z, off, run(T, E, k, router, z, picks(z, k), off))


@pytest.mark.parametrize("T,n_seq", [(16384, 1), (9000, 2), (4096, 1), (4095, 1), (40000, 3)])
def test_long_sequences_are_counted_in_parts(T, n_seq):
    E, k = 8, 2
    z = np.random.default_rng(T).standard_normal((T, E)).astype(np.float32)
    off = [0] + [T * (i + 1) // n_seq - 3 for i in range(n_seq)]
    check(T, E, k, "softmax", z, off, run(T, E, k, "softmax", z, picks(z, k), off))


@pytest.mark.parametrize("router", ["norm", "softmax"])
def test_padding_is_not_read_and_gets_no_gradient(router):
    T, E, k = 50, 16, 2
    z = np.random.default_rng(9).standard_normal((T, E)).astype(np.float32)
    idx, off = picks(z, k), [4, 20, 20, 41]
    want = run(T, E, k, router, z, idx, off)
    zp, ip = z.copy(), idx.copy()
    zp[:4], zp[41:] = np.nan, np.inf
    ip[:4], ip[41:] = -1, 1 << 30
    got = run(T, E, k, router, zp, ip, off)
    for a, b in zip(got, want):
        assert np.array_equal(host(a), host(b))
    assert not host(got[2])[:4].any() and not host(got[2])[41:].any()


def test_offsets_outside_the_tokens_are_cut_off_and_all_sequences_may_be_empty():
    T, E, k = 20, 8, 2
    z = np.random.default_rng(10).standard_normal((T, E)).astype(np.float32)
    check(T, E, k, "norm", z, [-5, 6, 90], run(T, E, k, "norm", z, picks(z, k), [-5, 6, 90]))
    counts, loss, dz, ds = run(T, E, k, "norm", z, picks(z, k), [7, 7, 7])
    assert not host(counts).any() and host(loss)[0] == 0 and not host(dz).any() and host(ds)[0] == 0
    z[3] = 0.0                                                     # a token without a direction: no gradient, no NaN
    check(T, E, k, "norm", z, [0, T], run(T, E, k, "norm", z, picks(z, k), [0, T]))


def test_without_gradients_and_at_any_address():
    T, E, k = 77, 24, 3
    z = np.random.default_rng(11).standard_normal((T, E)).astype(np.float32)
    off = [0, 30, 77]
    want = run(T, E, k, "norm", z, picks(z, k), off)
    got = run(T, E, k, "norm", z, picks(z, k), off, grad=False)
    assert np.array_equal(host(got[0]), host(want[0])) and host(got[1])[0] == host(want[1])[0]
    check(T, E, k, "norm", z, off, run(T, E, k, "norm", z, picks(z, k), off, shift=1))


@pytest.mark.parametrize("dtype,T,d,E,k,router", [("f32", 60, 40, 9, 2, "norm"), ("f32", 500, 64, 16, 2, "softmax"), ("bf16", 300, 128, 24, 3, "norm"),
                                                   ("bf16", 400, 128, 30, 2, "softmax"), ("bf16", 70, 64, 512, 8, "norm")])
def test_router_backward_takes_the_gradients_in(dtype, T, d, E, k, router):
    """The sum of both losses through one call; with none given the bits of the call without them."""
    import torch
    from oracle import unipool_oracle as P
    from tests.gpu_util import TOL, rel_err, round_act
    U = lib()
    g = np.random.default_rng(12)
    x, w = round_act(g.standard_normal((T, d)), dtype), round_act(g.standard_normal((E, d)) / (np.sqrt(d) if router == "softmax" else 1), dtype)
    dgate, coef = g.standard_normal((T, k)).astype(np.float32), (0.1 * g.standard_normal(E)).astype(np.float32)
    z = P.router_logits(x, w).astype(np.float32)
    idx, off = picks(z, k), [0, T // 3, T - 5]
    sh = shape(T, E, k, router, d)
    sh.dtype = U.BF16 if dtype == "bf16" else U.F32
    ws = torch.empty(U.workspace_bytes(sh), dtype=torch.uint8, device="cuda")
    gx, gw, gz, gi, gd, gc = dev(x, dtype), dev(w, dtype), dev(z), dev(idx), dev(dgate), dev(coef)
    counts, loss, dz, ds = (torch.zeros(n, dtype=t, device="cuda") for n, t in (((2, E), torch.int32), (1, torch.float32), ((T, E), torch.float32), (1, torch.float32)))
    U.seq_balance_loss(sh, 2, dev(np.asarray(off, np.int32)), 40.0, gz, gi, counts, loss, dz, ds, ws)

    def backward(add):
        out = [torch.zeros((E, d), device="cuda"), torch.zeros(1, device="cuda"), torch.zeros_like(gx)]
        if add is None:
            U.route_bwd(sh, gx, gw, gz, gi, gd, gc, *out, False, ws)
        else:
            U.route_bwd_add(sh, gx, gw, gz, gi, gd, gc, *add, *out, False, ws)
        torch.cuda.synchronize()
        return out
    for a, b in zip(backward(None), backward((None, None))):
        assert torch.equal(a, b)
    _, _, dz_ref, ds_ref = O.seq_balance_loss(z, idx, off, 40.0, router, SIGMA, CC, EPS)
    own = P.route_bwd(x, w, z.astype(np.float64), idx, dgate, coef, SIGMA, CC, EPS, router=router)
    dw_own, ds_own, dx_own = (own[n] for n in ("dw_router", "d_sigma", "dx")) if isinstance(own, dict) else (own[1], own[2], own[0])
    dw, dsig, dx = (host(t) for t in backward((dz, ds)))
    assert rel_err(dw, dw_own + dz_ref.T @ x) <= TOL[dtype]
    assert rel_err(dx, dx_own + dz_ref @ w) <= TOL[dtype]
    total = np.asarray(ds_own).reshape(-1)[0] + ds_ref
    assert abs(dsig[0] - total) <= 1e-5 * max(abs(total), np.abs(dgate).sum())


@pytest.mark.parametrize("T,E,n_seq", [(256, 32, 256), (257, 32, 256), (256, 33, 256), (256, 512, 16), (256, 512, 17), (100, 8, 3000)])
def test_one_workgroup_and_several(T, E, n_seq):
    """Both sides of the line up to which a single workgroup does everything, and more sequences than tokens."""
    k = 2
    z = np.random.default_rng(E + n_seq).standard_normal((T, E)).astype(np.float32)
    off = np.sort(np.random.default_rng(n_seq).integers(0, T + 1, n_seq + 1)).astype(np.int32)
    for router in ("norm", "softmax"):
        check(T, E, k, router, z, off, run(T, E, k, router, z, picks(z, k), off))


@pytest.mark.parametrize("router", ["norm", "softmax"])
def test_many_empty_sequences_between_those_with_tokens(router):
    T, E, k = 310, 16, 2
    z = np.random.default_rng(12).standard_normal((T, E)).astype(np.float32)
    off = [0] * 700 + [1, 2, 2, 3] + [7] * 1500 + [100] * 3 + [101, 150] + [151] * 900 + [300] * 2
    check(T, E, k, router, z, off, run(T, E, k, router, z, picks(z, k), off))


@pytest.mark.parametrize("T,E", [(20, 8), (400, 70)])
@pytest.mark.parametrize("tiny", [0.0, 1e-30])
def test_tokens_without_a_direction_and_without_eps(T, E, tiny, monkeypatch):
    """Logits that are all zero, or so small that their squares are: no part of loss and gradients, where 1 / norm is infinite.  The
    router's backward pass takes the gradients of a batch with zero logits in."""
    import sys

    import torch
    monkeypatch.setattr(sys.modules[__name__], "EPS", 0.0)
    k = 2
    z = np.random.default_rng(T).standard_normal((T, E)).astype(np.float32)
    z[3], z[T - 1] = 0.0, tiny
    off = [0, T // 2, T]
    got = run(T, E, k, "norm", z, picks(z, k), off)
    zr = np.where(np.abs(z) < 1e-20, 0.0, z)                       # what the squares in float make of them
    c_ref, l_ref, dz_ref, ds_ref = O.seq_balance_loss(zr, picks(z, k), off, ALPHA, "norm", SIGMA, CC, EPS)
    assert np.array_equal(host(got[0]), c_ref)
    assert abs(host(got[1])[0] - l_ref) <= C * abs(l_ref) and abs(host(got[3])[0] - ds_ref) <= C * abs(ds_ref)
    assert np.isfinite(host(got[2])).all() and not host(got[2])[[3, T - 1]].any()
    if tiny:                                                       # (its score itself is infinite: relu(z) / 0)
        return
    U, d = lib(), 64
    sh = shape(T, E, k, "norm", d)
    ws = torch.empty(U.workspace_bytes(sh), dtype=torch.uint8, device="cuda")
    x, w, dgate = torch.randn(T, d, device="cuda"), torch.randn(E, d, device="cuda"), torch.ones(T, k, device="cuda")
    out = []
    for extra in ((None, None), (got[2], got[3])):
        dw, ds, dx = torch.zeros(E, d, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(T, d, device="cuda")
        U.route_bwd_add(sh, x, w, dev(z), dev(picks(z, k)), dgate, None, *extra, dw, ds, dx, False, ws)
        out.append((dw, ds, dx))
    assert all(torch.isfinite(t).all() for o in out for t in o)
    # sigma's own gradient is a sum of k T terms, the scores over sigma
    scores = float(host(out[0][1])[0])
    assert abs(float(host(out[1][1])[0]) - scores - ds_ref) <= C * (abs(scores) + CC * k * T + abs(ds_ref))


def test_counts_of_many_sequences_in_parts_past_30_bits_of_tokens():
    """Tokens and the tokens that a round of workgroups counts pass 2^31 together.  One expert with one pick a token: counts are the lengths,
    every score is 1, the loss alpha."""
    import torch
    U, T, n_seq = lib(), 1_200_000_000, 250_000
    sh = shape(T, 1, 1, "softmax")
    z, idx = torch.zeros((T, 1), device="cuda"), torch.zeros((T, 1), dtype=torch.int32, device="cuda")
    off = torch.arange(n_seq + 1, device="cuda").mul_(4800).int()
    off[-1] = T
    off[1:-1] += torch.randint(-2000, 2000, (n_seq - 1,), device="cuda").int()
    ws = torch.empty(U.workspace_bytes(sh), dtype=torch.uint8, device="cuda")
    counts, loss = torch.full((n_seq, 1), -1, dtype=torch.int32, device="cuda"), torch.full((1,), float("nan"), device="cuda")
    U.seq_balance_loss(sh, n_seq, off, ALPHA, z, idx, counts, loss, None, None, ws)
    torch.cuda.synchronize()
    assert torch.equal(counts[:, 0], off[1:] - off[:-1])
    # a wavefront adds the shares of its tokens one after the other, 16 lanes' groups of them; then 16 wavefronts and 512 workgroups
    assert abs(float(loss) - ALPHA) <= (T / (512 * 16 * 4) + 64) * 2.0 ** -24 * ALPHA
