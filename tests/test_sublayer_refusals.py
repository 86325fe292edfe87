"""Calls of the operators around the pool layer that are refused, on the host and before anything is launched."""
import pytest


@pytest.fixture(scope="module")
def U():
    import __graft_entry__ as g
    g.ensure_built()
    import paper_2605_06665_amd as U
    U.load_library()
    return U


P = 1 << 20            # an address aligned to everything; nothing is launched, so nothing reads it


def shape(U, **kw):
    base = dict(T=128, d_model=64, d_ff=128, E=8, k=2, L=2, dtype=U.BF16, sigma=1.0, c=2.5, eps=1e-6, alpha_pool=0.01)
    base.update(kw)
    return U.Shape(**base)


class Ws:
    """A workspace that is only looked at."""
    def __init__(self, nbytes, ptr=P):
        self.nbytes, self.ptr = nbytes, ptr

    def data_ptr(self):
        return self.ptr


def ws(U, sh):
    return Ws(U.workspace_bytes(sh))


def test_norm(U):
    sh = shape(U)
    call = lambda sh=sh, x=P, r=None, w=P, eps=1e-6, h=P, y=P, q=None, s=None: U.rmsnorm(sh, x, r, w, eps, h, y, q, s, stream=0)  # noqa: E731
    for kw, msg in ((dict(x=None), "x is NULL"), (dict(w=None), "weight is NULL"), (dict(y=None), "neither y nor y_q"),
                    (dict(q=P), "y_q and y_scale"), (dict(s=P), "y_q and y_scale"), (dict(eps=-1e-6), "norm_eps"),
                    (dict(eps=float("nan")), "norm_eps"), (dict(sh=shape(U, T=0)), "positive"),
                    (dict(sh=shape(U, d_model=16448)), "d_model=16448"),
                    (dict(sh=shape(U, dtype=U.F32, d_model=48), q=P, s=P), "multiple of 32")):
        with pytest.raises(U.UniPoolError, match=msg):
            call(**kw)


def test_norm_backward(U):
    sh = shape(U)
    call = lambda sh=sh, h=P, w=P, dy=P, dh=None, eps=1e-6, dx=P, dw=P, ws=ws(U, sh): U.rmsnorm_bwd(sh, h, w, dy, dh, eps, dx, dw, ws, stream=0)  # noqa: E731
    for kw, msg in ((dict(h=None), "h is NULL"), (dict(w=None), "weight is NULL"), (dict(dy=None), "dy is NULL"),
                    (dict(dx=None), "dx is NULL"), (dict(dw=None), "d_weight is NULL"), (dict(eps=-1.0), "norm_eps"),
                    (dict(ws=None), "workspace is NULL"), (dict(ws=Ws(64)), "64 bytes"), (dict(ws=Ws(1 << 40, P + 4)), "aligned"),
                    (dict(sh=shape(U, d_model=16448)), "d_model=16448")):
        with pytest.raises(U.UniPoolError, match=msg):
            call(**kw)


def test_balance_loss(U):
    sh = shape(U)
    call = lambda n=3, off=P, z=P, idx=P, cnt=P, loss=P, ws=ws(U, sh): U.seq_balance_loss(sh, n, off, 0.1, z, idx, cnt, loss, None, None, ws, stream=0)  # noqa: E731
    for kw, msg in ((dict(n=0), "n_seq=0"), (dict(n=-1), "n_seq=-1"), (dict(n=(1 << 20) + 1), "n_seq="), (dict(off=None), "seq_offsets is NULL"),
                    (dict(z=None), "logits is NULL"), (dict(idx=None), "topk_idx is NULL"), (dict(cnt=None), "counts is NULL"),
                    (dict(loss=None), "loss is NULL"), (dict(ws=None), "workspace is NULL"), (dict(ws=Ws(64)), "64 bytes")):
        with pytest.raises(U.UniPoolError, match=msg):
            call(**kw)


def test_router_backward_with_further_gradients(U):
    sh = shape(U)
    names = ("x", "w_router", "logits", "topk_idx", "dgate", "aux_coef", "d_logits", "d_sigma_in", "d_w_router", "d_sigma", "dx")
    for n in names:
        if n not in ("aux_coef", "d_logits", "d_sigma_in"):
            with pytest.raises(U.UniPoolError, match="%s is NULL" % n):
                U.route_bwd_add(sh, *[None if m == n else P for m in names], False, ws(U, sh), stream=0)
    with pytest.raises(U.UniPoolError, match="workspace"):
        U.route_bwd_add(sh, *[P] * len(names), False, None, stream=0)


def test_quantize(U):
    call = lambda dt=U.BF16, rows=4, cols=64, src=P, q=P, s=P: U.quantize_mx8(dt, rows, cols, src, q, s, stream=0)  # noqa: E731
    for kw, msg in ((dict(dt=2), "dtype 2"), (dict(rows=0), "rows"), (dict(cols=0), "cols"), (dict(cols=48), "multiple of 32"),
                    (dict(cols=-32), "cols"), (dict(rows=1 << 41), "too large"), (dict(rows=1 << 36, cols=1 << 13), "too large"),
                    (dict(src=None), "src is NULL"), (dict(q=None), "q is NULL"), (dict(s=None), "scale is NULL")):
        with pytest.raises(U.UniPoolError, match=msg):
            call(**kw)


def test_experts(U):
    sh = shape(U)
    names = ("x_q", "x_scale", "slot_of_row", "expert_offsets", "w_gate_up_q", "w_gate_up_scale", "w_down_q", "w_down_scale", "h_q", "h_scale",
             "y_perm")

    def call(sh=sh, ws=ws(U, sh), **kw):
        U.expert_ffn_fwd_mx8(sh, *[kw.get(n, P) for n in names], ws, stream=0)
    for n in names:
        if n != "slot_of_row":
            with pytest.raises(U.UniPoolError, match="%s is NULL" % n):
                call(**{n: None})
    for n in ("x_q", "w_gate_up_q", "w_down_q", "h_q", "y_perm"):
        with pytest.raises(U.UniPoolError, match="aligned to 16"):
            call(**{n: P + 8})
    for n in ("x_scale", "w_gate_up_scale", "w_down_scale", "h_scale"):
        with pytest.raises(U.UniPoolError, match="aligned to 4"):
            call(**{n: P + (8 if n[0] == "w" else 2)})
    with pytest.raises(U.UniPoolError, match="bfloat16 mode only"):
        call(sh=shape(U, dtype=U.F32))
    with pytest.raises(U.UniPoolError, match="multiples of 64"):
        call(sh=shape(U, d_ff=96))
    big = shape(U, T=1, E=1, k=1, d_ff=(1 << 20) + 64)
    with pytest.raises(U.UniPoolError, match="at most 2"):
        call(sh=big, ws=ws(U, big))
    for w, msg in ((None, "workspace is NULL"), (Ws(64), "64 bytes")):
        with pytest.raises(U.UniPoolError, match=msg):
            call(ws=w)


def test_binding_refuses_strided_tensors(U):
    import torch
    t = torch.zeros(8, 8)[:, ::2]
    with pytest.raises(U.UniPoolError, match="contiguous"):
        U.rmsnorm(shape(U), t, None, P, 1e-6, None, P, None, None, stream=0)


def test_limits_of_experts_and_conversion(U):
    with pytest.raises(U.UniPoolError, match="at most 2"):
        U.mx8_form(shape(U, T=1, E=1, k=1, d_ff=(1 << 20) + 64))
    with pytest.raises(U.UniPoolError, match="bfloat16 mode only"):
        U.mx8_form(shape(U, dtype=U.F32))
    for rows, cols in ((1 << 30, 32), (1 << 26, 2048)):        # 2^24 workgroups: more threads than a launch may have
        with pytest.raises(U.UniPoolError, match="too large"):
            U.quantize_mx8(U.BF16, rows, cols, P, P, P, stream=0)


def test_conversion_of_the_longest_rows(U):
    for cols in (2147483520 + 32, 2147483616):                 # 2^24 workgroups a row of 64, where cols + 127 passes 31 bits
        with pytest.raises(U.UniPoolError, match="too large"):
            U.quantize_mx8(U.BF16, 1, cols, P, P, P, stream=0)


def test_balance_loss_of_the_most_tokens(U):
    sh = shape(U, T=(1 << 31) - 63, k=1, E=1)
    with pytest.raises(U.UniPoolError, match="2\\^31 - 64"):
        U.seq_balance_loss(sh, 1, P, 0.1, P, P, P, P, None, None, Ws(1 << 60), stream=0)


def test_serving_refuses_weights_that_are_not_on_the_device(U):
    import torch
    from paper_2605_06665_amd.pipeline import PoolServe
    T, d, f, E, k = 8, 64, 64, 4, 2
    w = torch.zeros(E, 2 * f, d, dtype=torch.bfloat16), torch.zeros(E, d, f, dtype=torch.bfloat16)
    for bad in (w, (w[0].float(), w[1]), (w[0], w[1][:-1])):
        with pytest.raises(AssertionError):
            PoolServe(T, d, f, E, k, 2.5, 1e-6, *bad)
