"""The operators around the pool layer as they are used together: the residual stack of norms and layers forward and backward
(PoolStack), with the balance loss over sequences, and its forward pass for serving with the experts in 8 bits (PoolServe), against
float64 chains of the plain implementations.  Selections are discrete: the chain in float64 takes over the GPU's picks, which
are checked against its own logits."""
import numpy as np
import pytest

from oracle import sublayer_oracle as S
from oracle import unipool_oracle as O
from tests.gpu_util import TOL, dev, host, rel_err, round_act

pytestmark = pytest.mark.gpu

NORM_EPS, EPS, C = 1e-5, 1e-6, 2.3


def inputs(T, d, f, E, L, dtype, seed, scale=1.0):
    g = np.random.default_rng(seed)
    r = lambda *s, std=1.0: round_act(g.standard_normal(s) * std, dtype)  # noqa: E731
    return dict(x=r(T, d), norms=[round_act(1 + 0.1 * g.standard_normal(d), dtype) for _ in range(L + 1)], wrs=[r(E, d, std=scale) for _ in range(L)],
                wg=r(E, f, d, std=0.05), wu=r(E, f, d, std=0.05), wd=r(E, d, f, std=0.05), gy=r(T, d), sigmas=[1.0 + 0.1 * l for l in range(L)])


def chain(i, idxs, k, alpha, seq, router):
    """Forward and backward of the stack in float64; idxs: the picks.  seq: (offsets, alpha) or None."""
    L = len(i["wrs"])
    hs, ys, fws = [np.asarray(i["x"], np.float64)], [], []
    ys.append(S.rmsnorm(hs[0], None, i["norms"][0], NORM_EPS)[1])
    for l in range(L):
        fw = O.moe_layer_fwd(ys[l], i["wrs"][l], i["wg"], i["wu"], i["wd"], k, i["sigmas"][l], C, EPS, idxs[l], router)
        h, y = S.rmsnorm(fw["out"], hs[l], i["norms"][l + 1], NORM_EPS)
        fws.append(fw); hs.append(h); ys.append(y)
    counts, psum = np.stack([f["counts"] for f in fws]), np.stack([f["psum"] for f in fws])
    _, _, loss, coef = O.pool_aux_loss(counts, psum, len(i["x"]), k, alpha)
    dh, d_norm = S.rmsnorm_bwd(hs[L], i["norms"][L], i["gy"], None, NORM_EPS)
    d_norms, dwr, ds, seq_loss = [None] * L + [d_norm], [None] * L, [None] * L, []
    dwg, dwu, dwd = (np.zeros(i[n].shape) for n in ("wg", "wu", "wd"))
    for l in reversed(range(L)):
        bw = O.moe_layer_bwd(fws[l], ys[l], i["wrs"][l], i["wg"], i["wu"], i["wd"], dh, coef, k, i["sigmas"][l], C, EPS, router)
        dy, dwr[l], ds[l] = bw["dx"], bw["dw_router"], bw["dsigma"]
        if seq is not None:
            _, ls, dz, dsig = S.seq_balance_loss(fws[l]["z"], idxs[l], seq[0], seq[1], router, i["sigmas"][l], C, EPS)
            dy, dwr[l], ds[l] = dy + dz @ i["wrs"][l], dwr[l] + dz.T @ ys[l], ds[l] + dsig
            seq_loss.insert(0, ls)
        dwg += bw["dw_gate"]; dwu += bw["dw_up"]; dwd += bw["dw_down"]
        dh, d_norms[l] = S.rmsnorm_bwd(hs[l], i["norms"][l], dy, dh, NORM_EPS)
    return dict(y=ys[L], hs=hs, fws=fws, loss=loss, seq_loss=seq_loss, dx=dh, d_norm=np.stack(d_norms), dwr=dwr, ds=ds,
                dwgu=np.concatenate([dwg, dwu], axis=1), dwd=dwd)


def pick_slack(dtype):
    # a pick may differ from the chain's own where logits are nearer than the rounding of the stack's activations
    return 1e-4 if dtype == "f32" else 6e-2


@pytest.mark.parametrize("dtype,T,d,f,E,k,L,router,wgrad,n_seq", [
    ("f32", 90, 40, 56, 7, 2, 3, "norm", "pool", 4), ("f32", 130, 64, 48, 8, 1, 2, "softmax", "layer", None),
    ("bf16", 300, 128, 192, 16, 2, 3, "norm", "pool", 5), ("bf16", 260, 192, 128, 12, 3, 2, "softmax", "layer", 3)])
def test_stack_forward_and_backward(dtype, T, d, f, E, k, L, router, wgrad, n_seq):
    import torch
    import paper_2605_06665_amd as U
    from paper_2605_06665_amd.pipeline import PoolStack, PoolStep
    i = inputs(T, d, f, E, L, dtype, T, 1.0 if router == "norm" else 2.0 / np.sqrt(d))
    alpha, seq_alpha = 0.02, 0.5
    ps = PoolStep(T, d, f, E, k, L, U.BF16 if dtype == "bf16" else U.F32, C, EPS, alpha, wgrad=wgrad, router=router, n_seq=n_seq,
                  seq_alpha=seq_alpha)
    seq = None
    if n_seq is not None:
        off = np.sort(np.random.default_rng(5).integers(2, T - 3, n_seq + 1)).tolist()
        off[1] = off[2]                                    # an empty sequence; tokens in front and behind belong to none
        ps.set_sequences(off)
        seq = (off, seq_alpha)
    st = PoolStack(ps, norm_eps=NORM_EPS)
    w = [dev(n, dtype) for n in i["norms"]], [dev(n, dtype) for n in i["wrs"]], i["sigmas"], dev(np.concatenate([i["wg"], i["wu"]], axis=1), dtype), dev(i["wd"], dtype)
    x = dev(i["x"], dtype)
    y = st.forward(x, *w)
    dx = st.backward(dev(i["gy"], dtype), *w)
    torch.cuda.synchronize()
    idxs = [host(l.topk_idx).astype(np.int64) for l in ps.layers]
    ref = chain(i, idxs, k, alpha, seq, router)
    for l in range(L):                                     # the picks are right for the chain's logits up to the rounding in front of them
        z = ref["fws"][l]["z"]
        zn = z / np.linalg.norm(z, axis=1, keepdims=True)
        kth = -np.sort(-zn, axis=1)[:, k - 1]
        assert (np.take_along_axis(zn, idxs[l], 1).min(axis=1) >= kth - pick_slack(dtype)).all()
    # bars of the whole step, per tensor, for a chain of L layers
    tol = TOL[dtype] * L * (10 if dtype == "f32" else 2)
    assert rel_err(host(y), ref["y"]) <= tol and rel_err(host(st.h[L]), ref["hs"][L]) <= tol
    assert rel_err(host(dx), ref["dx"]) <= tol and rel_err(host(st.d_norm), ref["d_norm"]) <= tol
    assert rel_err(host(ps.d_w_gate_up), ref["dwgu"]) <= tol and rel_err(host(ps.d_w_down), ref["dwd"]) <= tol
    for l in range(L):
        assert rel_err(host(ps.layers[l].d_w_router), ref["dwr"][l]) <= tol
        if n_seq is not None:
            assert abs(host(ps.seq_loss)[l] - ref["seq_loss"][l]) <= tol * abs(ref["seq_loss"][l])
            want = np.zeros((n_seq, E), np.int64)
            for b in range(n_seq):
                want[b] = np.bincount(idxs[l][seq[0][b]:seq[0][b + 1]].reshape(-1), minlength=E)
            assert np.array_equal(host(ps.seq_counts)[l], want)
    assert torch.equal(x, dev(i["x"], dtype))


def test_steps_without_sequences_are_unchanged_and_with_coefficient_zero_the_same():
    import torch
    import paper_2605_06665_amd as U
    from paper_2605_06665_amd.pipeline import PoolStep
    T, d, f, E, k, L = 300, 128, 192, 16, 2, 2
    i = inputs(T, d, f, E, L, "bf16", 9)
    args = ([dev(i["x"], "bf16")] * L, [dev(w, "bf16") for w in i["wrs"]], i["sigmas"], dev(np.concatenate([i["wg"], i["wu"]], axis=1), "bf16"),
            dev(i["wd"], "bf16"), [dev(i["gy"], "bf16")] * L)
    res = []
    for kw in ({}, dict(n_seq=4, seq_alpha=0.0)):
        ps = PoolStep(T, d, f, E, k, L, U.BF16, C, EPS, 0.02, **kw)
        ps.step(*args)
        torch.cuda.synchronize()
        res.append([ps.d_w_gate_up, ps.d_w_down, ps.loss] + [t for l in ps.layers for t in (l.out, l.dx, l.d_w_router, l.d_sigma)])
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_recorded_step_with_sequences():
    import torch
    import paper_2605_06665_amd as U
    from paper_2605_06665_amd.pipeline import PoolStep
    T, d, f, E, k, L = 200, 128, 128, 8, 2, 2
    i = inputs(T, d, f, E, L, "bf16", 10)
    xs = [dev(i["x"], "bf16").clone() for _ in range(L)]
    args = (xs, [dev(w, "bf16") for w in i["wrs"]], i["sigmas"], dev(np.concatenate([i["wg"], i["wu"]], axis=1), "bf16"), dev(i["wd"], "bf16"),
            [dev(i["gy"], "bf16")] * L)
    ps = PoolStep(T, d, f, E, k, L, U.BF16, C, EPS, 0.02, n_seq=3, seq_alpha=0.3)
    graph = ps.capture(*args)
    for rep in range(3):
        xs[0].copy_(torch.roll(xs[0], rep, 0))
        ps.set_sequences([rep, 40 + rep, 40 + rep, 190])   # the graph reads the offsets in place
        ps.step(*args)
        torch.cuda.synchronize()
        outs = [ps.seq_loss, ps.seq_counts, ps.d_w_gate_up] + [t for l in ps.layers for t in (l.dx, l.d_w_router, l.seq_d_logits)]
        want = [t.clone() for t in outs]
        for t in outs:
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("T,n,d,f,E,k,L,router", [(64, 64, 128, 192, 8, 2, 3, "norm"), (40, 1, 192, 128, 12, 3, 2, "softmax"), (300, 257, 320, 192, 16, 2, 2, "norm")])
def test_serving_in_8_bits(T, n, d, f, E, k, L, router):
    """Layer by layer against the formulas on the GPU's own inputs of that layer (what 8 bits round differs from the bfloat16 stack on purpose),
    and the whole forward pass against those layers, eager and replayed."""
    import torch
    from paper_2605_06665_amd.pipeline import PoolServe
    i = inputs(T, d, f, E, L, "bf16", T + d, 1.0 if router == "norm" else 2.0 / np.sqrt(d))
    wgu, wd = np.concatenate([i["wg"], i["wu"]], axis=1), i["wd"]
    sv = PoolServe(T, d, f, E, k, C, EPS, dev(wgu, "bf16"), dev(wd, "bf16"), router=router, norm_eps=NORM_EPS)
    wguv = S.from_mx8(*S.to_mx8(wgu.reshape(-1, d))).reshape(wgu.shape)
    wdv = S.from_mx8(*S.to_mx8(wd.reshape(-1, f))).reshape(wd.shape)
    norms, wrs = [dev(w, "bf16") for w in i["norms"]], [dev(w, "bf16") for w in i["wrs"]]
    x = dev(i["x"][:n], "bf16")
    h, out = None, x
    for l in range(L):
        res = None if l == 0 else h
        hn = torch.empty_like(x)
        got = sv.layer(out, res, hn, norms[l], wrs[l], i["sigmas"][l]).clone()
        torch.cuda.synchronize()
        h_ref, y_ref = S.rmsnorm(host(out), None if res is None else host(res), i["norms"][l], NORM_EPS)
        assert rel_err(host(hn), h_ref) <= TOL["bf16"] and rel_err(host(sv.y[:n]), y_ref) <= TOL["bf16"]
        idx = host(sv.topk_idx[:n]).astype(np.int64)
        r = O.route(host(sv.y[:n]), i["wrs"][l], k, i["sigmas"][l], C, EPS, idx, router)
        r = r if isinstance(r, dict) else dict(gate=r[1])
        off, ros, sor = O.permutation(idx, E)
        scales = sv.x_q[1].view(-1)[:4 * n * -(-d // 128)].view(-1, n, 4)
        xv = S.from_mx8(sv.x_q[0][:n].cpu().numpy(), scales.cpu().numpy())
        assert np.linalg.norm(xv - y_ref) <= 0.04 * np.linalg.norm(y_ref)          # half a step of e4m3 at most, 2^-4
        hv = S.expert_h(xv[sor // k], off, wguv)
        y_rows = S.expert_y(S.from_mx8(*S.to_mx8(hv)), off, wdv)
        want = O.combine(y_rows, ros, host(sv.topk_gate[:n]).astype(np.float64))
        assert rel_err(host(got), want) <= TOL["bf16"]
        h, out = hn, got
    y_ref = S.rmsnorm(host(out), host(h), i["norms"][L], NORM_EPS)[1]
    y = sv.forward(x, norms, wrs, i["sigmas"]).clone()
    assert rel_err(host(y), y_ref) <= TOL["bf16"]
    assert torch.equal(x, dev(i["x"][:n], "bf16"))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        yg = sv.forward(x, norms, wrs, i["sigmas"])
    for rep in range(3):
        x.copy_(torch.roll(x, 1, 0))
        want = sv.forward(x, norms, wrs, i["sigmas"]).clone()
        yg.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(yg, want)


def test_serving_takes_its_own_result_and_refuses_what_does_not_fit():
    import torch
    from paper_2605_06665_amd.pipeline import PoolServe
    T, d, f, E, k, L = 20, 128, 64, 4, 2, 2
    i = inputs(T, d, f, E, L, "bf16", 5)
    sv = PoolServe(T, d, f, E, k, C, EPS, dev(np.concatenate([i["wg"], i["wu"]], axis=1), "bf16"), dev(i["wd"], "bf16"), norm_eps=NORM_EPS)
    norms, wrs = [dev(w, "bf16") for w in i["norms"]], [dev(w, "bf16") for w in i["wrs"]]
    x = dev(i["x"], "bf16")
    first = sv.forward(x, norms, wrs, i["sigmas"]).clone()
    want = sv.forward(first, norms, wrs, i["sigmas"]).clone()
    assert torch.equal(sv.forward(sv.forward(x, norms, wrs, i["sigmas"]), norms, wrs, i["sigmas"]), want)
    for bad in (lambda: sv.forward(x, norms, [], []), lambda: sv.forward(x, norms, wrs, i["sigmas"][:1]), lambda: sv.forward(x, norms[:L], wrs, i["sigmas"]),
                lambda: sv.forward(x.float(), norms, wrs, i["sigmas"]), lambda: sv.forward(torch.cat([x, x]), norms, wrs, i["sigmas"])):
        with pytest.raises(AssertionError):
            bad()


def test_stack_refuses_its_result_as_its_input():
    import torch
    from paper_2605_06665_amd.pipeline import PoolStack, PoolStep
    from paper_2605_06665_amd import binding as B
    T, d, f, E, k, L = 20, 64, 64, 4, 2, 1
    i = inputs(T, d, f, E, L, "bf16", 6)
    stack = PoolStack(PoolStep(T, d, f, E, k, L, B.BF16, C, EPS, 0.01), NORM_EPS)
    args = ([dev(w, "bf16") for w in i["norms"]], [dev(w, "bf16") for w in i["wrs"]], i["sigmas"], dev(np.concatenate([i["wg"], i["wu"]], axis=1), "bf16"),
            dev(i["wd"], "bf16"))
    y = stack.forward(dev(i["x"], "bf16"), *args)
    with pytest.raises(AssertionError, match="kept for the backward"):
        stack.forward(y, *args)
    torch.cuda.synchronize()


@pytest.mark.parametrize("d,L", [(128, 1), (2112, 1), (8256, 1), (2112, 3)])
def test_serving_takes_its_own_result_with_any_number_of_layers(d, L):
    """With one layer the last norm finds the residual where its result goes; rows of one, four and sixteen wavefronts."""
    import torch
    from paper_2605_06665_amd.pipeline import PoolServe
    T, f, E, k = 20, 64, 4, 2
    i = inputs(T, d, f, E, L, "bf16", 5)
    sv = PoolServe(T, d, f, E, k, C, EPS, dev(np.concatenate([i["wg"], i["wu"]], axis=1), "bf16"), dev(i["wd"], "bf16"), norm_eps=NORM_EPS)
    w = [dev(n, "bf16") for n in i["norms"]], [dev(n, "bf16") for n in i["wrs"]], i["sigmas"]
    x = dev(i["x"], "bf16")
    for n in (T, 3, 1):
        want = x[:n].clone()
        for _ in range(3):
            want = sv.forward(want, *w).clone()
        got = x[:n].clone()
        for _ in range(3):
            got = sv.forward(got, *w)
        assert torch.equal(got, want)


@pytest.mark.parametrize("L", [1, 2])
def test_serving_takes_rows_of_its_own_result(L):
    """Rows of the result as the next call's x: with one layer it is read while the result goes out over it."""
    import torch
    from paper_2605_06665_amd.pipeline import PoolServe
    T, d, f, E, k = 900, 128, 64, 4, 2
    i = inputs(T, d, f, E, L, "bf16", 5)
    sv = PoolServe(T, d, f, E, k, C, EPS, dev(np.concatenate([i["wg"], i["wu"]], axis=1), "bf16"), dev(i["wd"], "bf16"), norm_eps=NORM_EPS)
    w = [dev(n, "bf16") for n in i["norms"]], [dev(n, "bf16") for n in i["wrs"]], i["sigmas"]
    x = dev(i["x"], "bf16")
    for lo, hi in ((1, T), (T - 1, T), (300, 700), (0, 5)):
        want = sv.forward(sv.forward(x, *w)[lo:hi].clone(), *w).clone()
        assert torch.equal(sv.forward(sv.forward(x, *w)[lo:hi], *w), want)


def test_serving_refuses_what_does_not_fit_argument_by_argument():
    import torch
    from paper_2605_06665_amd.pipeline import PoolServe
    T, d, f, E, k, L = 20, 128, 64, 4, 2, 2
    i = inputs(T, d, f, E, L, "bf16", 5)
    sv = PoolServe(T, d, f, E, k, C, EPS, dev(np.concatenate([i["wg"], i["wu"]], axis=1), "bf16"), dev(i["wd"], "bf16"), norm_eps=NORM_EPS)
    norms, wrs = [dev(n, "bf16") for n in i["norms"]], [dev(n, "bf16") for n in i["wrs"]]
    x = dev(i["x"], "bf16")
    r, h = torch.zeros_like(x), torch.empty_like(x)
    good = dict(x=x, residual=r, h=h, norm_weight=norms[0], w_router=wrs[0], sigma=1.0)
    for name, bad in (("x", x[:, :64].contiguous()), ("x", x.float()), ("x", x.cpu()), ("x", x[:0]), ("residual", r[:-1]), ("residual", r.float()), ("residual", r.cpu()),
                      ("h", h[:-1]), ("h", h.float()), ("h", sv.out), ("h", sv.out[:T]), ("norm_weight", norms[0].float()), ("norm_weight", norms[0][:-1]),
                      ("norm_weight", norms[0].cpu()), ("w_router", wrs[0].float()), ("w_router", wrs[0][:-1]), ("w_router", wrs[0].T.contiguous())):
        with pytest.raises(AssertionError):
            sv.layer(**{**good, name: bad})
    out = sv.layer(**good)
    with pytest.raises(AssertionError, match="two layers"):      # layer 0's output goes where this one lies, and layer 1 adds x to it
        sv.forward(out, norms, wrs, i["sigmas"])
    with pytest.raises(AssertionError):
        sv.forward(x, norms[:L] + [norms[L].float()], wrs, i["sigmas"])
    # what layer() does take: its output as the next one's x and residual
    want = sv.layer(out.clone(), out.clone(), h, norms[1], wrs[1], 1.0).clone()
    out = sv.layer(**good)
    assert torch.equal(sv.layer(out, out, h, norms[1], wrs[1], 1.0), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_stack_refuses_what_does_not_fit_argument_by_argument(dtype):
    import torch
    from paper_2605_06665_amd.pipeline import PoolStack, PoolStep
    from paper_2605_06665_amd import binding as B
    T, d, f, E, k, L = 20, 64, 64, 4, 2, 2
    i = inputs(T, d, f, E, L, dtype, 6)
    stack = PoolStack(PoolStep(T, d, f, E, k, L, B.BF16 if dtype == "bf16" else B.F32, C, EPS, 0.01), NORM_EPS)
    other = torch.float32 if dtype == "bf16" else torch.bfloat16
    x, norms, wrs = dev(i["x"], dtype), [dev(n, dtype) for n in i["norms"]], [dev(n, dtype) for n in i["wrs"]]
    pool = dev(np.concatenate([i["wg"], i["wu"]], axis=1), dtype), dev(i["wd"], dtype)
    good = dict(x=x, norm_weights=norms, w_routers=wrs, sigmas=i["sigmas"], w_gate_up=pool[0], w_down=pool[1])
    stack.forward(**good)
    dx = stack.backward(x, *list(good.values())[1:])
    for name, bad in (("x", x[:-1]), ("x", x.to(other)), ("x", x.cpu()), ("x", dx), ("x", stack.y[0]), ("x", stack.h[1]), ("norm_weights", norms[:L]),
                      ("norm_weights", norms[:L] + [norms[L].to(other)]), ("norm_weights", [norms[0][:-1]] + norms[1:]), ("w_routers", wrs[:1]),
                      ("w_routers", [wrs[0], wrs[1][:-1]]), ("w_routers", [wrs[0].to(other), wrs[1]]), ("sigmas", i["sigmas"][:1])):
        with pytest.raises(AssertionError):
            stack.forward(**{**good, name: bad})
        if name != "x":
            with pytest.raises(AssertionError):
                stack.backward(**{("grad_y" if n == "x" else n): v for n, v in {**good, name: bad}.items()})
    for bad in (x[:-1], x.to(other), x.cpu()):
        with pytest.raises(AssertionError):
            stack.backward(bad, *list(good.values())[1:])
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_stack_refuses_a_pool_that_does_not_fit(dtype):
    import torch
    from paper_2605_06665_amd.pipeline import PoolStack, PoolStep
    from paper_2605_06665_amd import binding as B
    T, d, f, E, k, L = 20, 64, 128, 4, 2, 1
    i = inputs(T, d, f, E, L, dtype, 6)
    stack = PoolStack(PoolStep(T, d, f, E, k, L, B.BF16 if dtype == "bf16" else B.F32, C, EPS, 0.01), NORM_EPS)
    other = torch.float32 if dtype == "bf16" else torch.bfloat16
    x, norms, wrs = dev(i["x"], dtype), [dev(n, dtype) for n in i["norms"]], [dev(n, dtype) for n in i["wrs"]]
    gu, down = dev(np.concatenate([i["wg"], i["wu"]], axis=1), dtype), dev(i["wd"], dtype)
    stack.forward(x, norms, wrs, i["sigmas"], gu, down)
    for pool in ((gu[:-1], down), (gu[:, :f].contiguous(), down), (gu.to(other), down), (gu.cpu(), down), (gu, down[:-1]), (gu, down.to(other)),
                 (gu, down.cpu()), (gu, down.transpose(1, 2).contiguous()), (down, gu)):
        for call in (stack.forward, stack.backward):
            with pytest.raises(AssertionError):
                call(x, norms, wrs, i["sigmas"], *pool)
    stack.backward(x, norms, wrs, i["sigmas"], gu, down)
    torch.cuda.synchronize()
