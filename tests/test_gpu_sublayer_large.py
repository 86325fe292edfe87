"""The operators around the pool layer where offsets pass 32 bits, on several streams at once, and as one recorded pass.  The calls'
results are compared bit for bit with calls on the last rows alone, calls alone and eager calls."""
import numpy as np
import pytest

from tests.gpu_util import dev

pytestmark = pytest.mark.gpu


def lib():
    import paper_2605_06665_amd as U
    return U


def shape(T, d, f=64, E=8, k=2, dtype=None, **kw):
    U = lib()
    return U.Shape(T=T, d_model=d, d_ff=f, E=E, k=k, L=1, dtype=U.BF16 if dtype is None else dtype, sigma=1.3, c=2.5, eps=1e-6, alpha_pool=0.01, **kw)


def ws(sh):
    import torch
    return torch.full((lib().workspace_bytes(sh),), 255, dtype=torch.uint8, device="cuda")


def u8(*s):
    import torch
    return torch.zeros(s, dtype=torch.uint8, device="cuda")


def mx8(v):
    U = lib()
    q, s = u8(*v.shape), u8(*U.mx8_scale_shape(*v.shape))
    U.quantize_mx8(U.BF16, *v.shape, v, q, s)
    return q, s


def test_norm_and_layout_past_32_bits():
    import torch
    U, T, d, n = lib(), 270001, 8192, 300                  # 2.2e9 values
    x = torch.randn(T, d, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(d, device="cuda").bfloat16()
    y, q, s = torch.empty_like(x), u8(T, d), u8(*U.mx8_scale_shape(T, d))
    U.rmsnorm(shape(T, d), x, None, w, 1e-6, None, y, q, s)
    xs = x[-n:].clone()
    y2, q2, s2 = torch.empty_like(xs), u8(n, d), u8(*U.mx8_scale_shape(n, d))
    U.rmsnorm(shape(n, d), xs, None, w, 1e-6, None, y2, q2, s2)
    assert torch.equal(y[-n:], y2) and torch.equal(q[-n:], q2) and torch.equal(s[:, -n:], s2)
    U.quantize_mx8(U.BF16, T, d, y, q, s)
    q2, s2 = mx8(y2)
    assert torch.equal(q[-n:], q2) and torch.equal(s[:, -n:], s2)
    dx, dw = torch.empty_like(x), torch.empty(d, device="cuda")
    sh = shape(T, d)
    U.rmsnorm_bwd(sh, x, w, y, None, 1e-6, dx, dw, ws(sh))
    dx2 = torch.empty_like(xs)
    U.rmsnorm_bwd(shape(n, d), xs, w, y2, None, 1e-6, dx2, torch.empty_like(dw), ws(shape(n, d)))
    assert torch.equal(dx[-n:], dx2) and torch.isfinite(dw).all()


def test_balance_loss_past_32_bits():
    import torch
    U, T, E, k, n = lib(), 4300007, 512, 2, 1000           # 2.2e9 logits
    z = torch.randn(T, E, device="cuda")
    idx = torch.randint(0, E, (T, k), device="cuda", dtype=torch.int32)

    def run(zz, ii, off, alpha):
        m = zz.shape[0]
        sh = shape(m, 64, E=E, k=k, dtype=U.F32)
        B = len(off) - 1
        counts, loss, dz, ds = torch.empty((B, E), dtype=torch.int32, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(zz), torch.empty(1, device="cuda")
        U.seq_balance_loss(sh, B, dev(np.asarray(off, np.int32)), alpha, zz, ii, counts, loss, dz, ds, ws(sh))
        return counts, dz
    # the last sequence's gradient goes by the number of sequences and its own tokens
    c, dz = run(z, idx, [0, T - n, T], 1.0)
    c2, dz2 = run(z[-n:].clone(), idx[-n:].clone(), [0, n], 0.5)
    assert torch.equal(c[1], c2[0]) and torch.equal(dz[-n:], dz2)
    assert torch.equal(c[0], torch.bincount(idx[:-n].flatten(), minlength=E).int())


def test_experts_past_32_bits():
    import torch
    U, E, d, f, k, n = lib(), 200, 1536, 4096, 1, 40       # 2.5e9 bytes of gate-up weights
    wgu = torch.randn(E * 2 * f, d, device="cuda", dtype=torch.bfloat16) * 0.05
    wd = torch.randn(E * d, f, device="cuda", dtype=torch.bfloat16) * 0.05
    qgu, qd = mx8(wgu), mx8(wd)
    lgu, ld = mx8(wgu[-2 * f:].clone()), mx8(wd[-d:].clone())
    for T in (n, 6 * E):                                   # streamed weights and tiles
        xq = mx8(torch.randn(T, d, device="cuda", dtype=torch.bfloat16))
        per = 0 if T == n else 5                           # the last expert has what the others leave
        off = dev(np.asarray([i * per for i in range(E)] + [T], np.int32))
        sh = shape(T, d, f, E, k)
        y = torch.zeros(T, d, device="cuda", dtype=torch.bfloat16)
        U.expert_ffn_fwd_mx8(sh, *xq, None, off, *qgu, *qd, u8(T, f), u8(*U.mx8_scale_shape(T, f)), y, ws(sh))
        m = T - (E - 1) * per
        sh1 = shape(m, d, f, 1, 1)
        y1 = torch.zeros(m, d, device="cuda", dtype=torch.bfloat16)
        U.expert_ffn_fwd_mx8(sh1, xq[0][-m:].clone(), xq[1][:, -m:].clone(), None, dev(np.asarray([0, m], np.int32)), *lgu, *ld, u8(m, f),
                             u8(*U.mx8_scale_shape(m, f)), y1, ws(sh1))
        assert torch.equal(y[-m:], y1) and y1.abs().max() > 0


def test_two_streams_at_once():
    """Each with a workspace of its own: the results of either call alone."""
    import torch
    U = lib()
    T, d, f, E, k = 700, 256, 320, 24, 2
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()  # noqa: E731
    wgu, wd, w = mx8(rnd(E * 2 * f, d) * 0.05), mx8(rnd(E * d, f) * 0.05), rnd(d)
    off = torch.linspace(0, T * k, E + 1, device="cuda").int()
    seq = dev(np.asarray([0, 100, 450, T], np.int32))

    class Side:
        def __init__(self):
            self.sh = shape(T, d, f, E, k)
            self.ws, self.x, self.sor = ws(self.sh), rnd(T, d), torch.randperm(T * k, device="cuda", generator=g).int()
            self.y, self.dx, self.o = torch.empty_like(self.x), torch.empty_like(self.x), torch.empty(T * k, d, device="cuda", dtype=torch.bfloat16)
            self.q, self.h = (u8(T, d), u8(*U.mx8_scale_shape(T, d))), (u8(T * k, f), u8(*U.mx8_scale_shape(T * k, f)))
            self.z, self.idx = torch.randn(T, E, device="cuda", generator=g), torch.randint(0, E, (T, k), device="cuda", generator=g).int()
            self.dw, self.loss, self.ds = torch.empty(d, device="cuda"), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
            self.counts, self.dz = torch.empty((3, E), device="cuda", dtype=torch.int32), torch.empty(T, E, device="cuda")
            self.stream = torch.cuda.Stream()

        def run(self):
            U.rmsnorm(self.sh, self.x, None, w, 1e-6, None, self.y, *self.q)
            U.expert_ffn_fwd_mx8(self.sh, *self.q, self.sor, off, *wgu, *wd, *self.h, self.o, self.ws)
            U.seq_balance_loss(self.sh, 3, seq, 0.1, self.z, self.idx, self.counts, self.loss, self.dz, self.ds, self.ws)
            U.rmsnorm_bwd(self.sh, self.x, w, self.y, None, 1e-6, self.dx, self.dw, self.ws)

        def results(self):
            return [t.clone() for t in (self.y, *self.q, *self.h, self.o, self.counts, self.loss, self.dz, self.ds, self.dx, self.dw)]
    sides = Side(), Side()
    want = []
    for s in sides:
        s.run()
        want.append(s.results())
    torch.cuda.synchronize()
    for _ in range(4):
        for s in sides:
            with torch.cuda.stream(s.stream):
                for _ in range(3):
                    s.run()
        torch.cuda.synchronize()
        for s, r in zip(sides, want):
            assert all(torch.equal(a, b) for a, b in zip(s.results(), r))
        torch.cuda.synchronize()


def test_stack_forward_and_backward_as_a_graph():
    import torch
    from paper_2605_06665_amd.pipeline import PoolStack, PoolStep
    U = lib()
    T, d, f, E, k, L = 400, 192, 128, 16, 2, 3
    g = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()  # noqa: E731
    st = PoolStep(T, d, f, E, k, L, U.BF16, 2.3, 1e-6, 0.01, n_seq=5, seq_alpha=0.02)
    st.set_sequences([0, 90, 90, 200, 333, 390])
    stack = PoolStack(st, 1e-5)
    x, gy = rnd(T, d), rnd(T, d)
    args = ([rnd(d) for _ in range(L + 1)], [rnd(E, d) for _ in range(L)], [1.0, 1.1, 1.2], rnd(E, 2 * f, d) * 0.05, rnd(E, d, f) * 0.05)

    def step():
        stack.forward(x, *args)
        return stack.backward(gy, *args)

    def results():
        out = [stack.y[L], stack.dx, stack.d_norm, st.loss, st.seq_loss, st.seq_counts, st.d_w_gate_up, st.d_w_down]
        return [t.clone() for t in out + [s.d_w_router for s in st.layers] + [s.d_sigma for s in st.layers]]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(3):
        x.copy_(torch.roll(x, 1, 0))
        step()
        want = results()
        for t in (stack.y[L], stack.dx, stack.d_norm, st.seq_loss):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results(), want))
