"""Which rows the experts in 8 bits look up through slot_of_row, and that they find the right ones.

slot_of_row need not come from a dispatch here: a row of the group order is whatever slot it names, so the tests give rows any tokens."""
import numpy as np
import pytest

from tests.gpu_util import dev

pytestmark = pytest.mark.gpu


def lib():
    import paper_2605_06665_amd as U
    return U


def shape(T, E, d, f, k):
    U = lib()
    return U.Shape(T=T, d_model=d, d_ff=f, E=E, k=k, L=1, dtype=U.BF16, sigma=1.0, c=2.5, eps=1e-6, alpha_pool=0.01)


def mx8(rows, cols, gen, std, scatter=False):
    """Random values laid out in 8 bits; scatter: rows differ by up to 2^40, so that another row's scales are noticed."""
    import torch
    U = lib()
    v = torch.randn((rows, cols), device="cuda", generator=gen) * std
    if scatter:
        v *= torch.exp2(torch.randint(-20, 20, (rows, 1), device="cuda", generator=gen))
    q = torch.empty((rows, cols), dtype=torch.uint8, device="cuda"), torch.empty(U.mx8_scale_shape(rows, cols), dtype=torch.uint8, device="cuda")
    U.quantize_mx8(U.F32, rows, cols, v, *q)
    return q


def run(T, E, d, f, k, rows, off, wgu, wd):
    import torch
    U, sh = lib(), shape(T, E, d, f, k)
    S = T * k
    ws = torch.full((U.workspace_bytes(sh),), 255, dtype=torch.uint8, device="cuda")
    hq = torch.full((S, f), 0x55, dtype=torch.uint8, device="cuda")
    hs = torch.full(U.mx8_scale_shape(S, f), 254, dtype=torch.uint8, device="cuda")
    y = torch.full((S, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    U.expert_ffn_fwd_mx8(sh, *rows, off, *wgu, *wd, hq, hs, y, ws)
    torch.cuda.synchronize()
    return hq, hs, y, ws


def in_group_order(x, slots, k):
    tok = slots.long() // k
    return x[0][tok].contiguous(), x[1][:, tok].contiguous(), None


# weights streamed to registers, tiles, and so many rows that their scales are brought into group order first
@pytest.mark.parametrize("T,E,d,f,k", [(5, 4, 128, 192, 2), (300, 4, 128, 192, 2), (300, 4, 448, 192, 2), (16384, 16, 384, 4096, 2)])
def test_slots_of_rows_outside_the_offsets_are_not_looked_up(T, E, d, f, k):
    """Token 0 belongs to the rows outside only, and its words of scales are found nowhere else: nothing may copy them."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(T)
    x, wgu, wd = mx8(T, d, g, 1.0), mx8(E * 2 * f, d, g, 0.05), mx8(E * d, f, g, 0.05)
    mark = torch.tensor([201, 17, 202, 18], dtype=torch.uint8, device="cuda")
    x[1][:, 0] = mark
    S = T * k
    lo, hi = S // 5, S - S // 4
    slots = torch.randint(k, S, (S,), device="cuda", generator=g).int()      # of tokens 1 ..
    slots[:lo], slots[hi:] = 0, 1                                            # of token 0
    off = dev(np.linspace(lo, hi, E + 1).astype(np.int32))
    got = run(T, E, d, f, k, (*x, slots), off, wgu, wd)
    want = run(T, E, d, f, k, in_group_order(x, slots, k), off, wgu, wd)
    for a, b in zip(got[:1] + got[2:3], want[:1] + want[2:3]):
        assert torch.equal(a[lo:hi].view(torch.uint8), b[lo:hi].view(torch.uint8))
    assert torch.equal(got[1][:, lo:hi], want[1][:, lo:hi])
    for r in (slice(0, lo), slice(hi, None)):
        assert (got[0][r] == 0x55).all() and (got[1][:, r] == 254).all() and torch.isnan(got[2][r]).all()
    words = got[3][:got[3].numel() // 4 * 4].view(torch.int32)
    assert not (words == mark.view(torch.int32)).any()


# (weights streamed, then) every tile form whose rows pass through LDS (three stages of 128 indices or more): below and above the limit from
# which scales are brought into group order first; three stages, where the look-up is just in time, and seven of which the last is half
@pytest.mark.parametrize("form,first,T,E,d,f,k", [
    (0, False, 12, 6, 448, 256, 2), (64128, False, 180, 9, 448, 192, 2), (96128, False, 1500, 5, 384, 256, 4), (64256, False, 1344, 128, 384, 4224, 2),
    (128256, False, 3200, 64, 384, 4096, 2), (128256, True, 6720, 134, 832, 4096, 2),
    (192256, False, 8192, 16, 384, 4096, 2), (192256, False, 8192, 12, 832, 2112, 3), (192256, True, 16384, 16, 384, 4160, 2), (192256, True, 9001, 10, 832, 4096, 3),
    (192256, False, 38400, 512, 448, 64, 2)])
def test_every_row_of_wide_tiles_is_the_one_looked_up(form, first, T, E, d, f, k):
    """All rows against rows in group order, bit for bit; rows spread over all the tiles of some experts against 64 bits."""
    import torch
    from oracle import sublayer_oracle as O
    U, S = lib(), T * k
    assert U.mx8_form(shape(T, E, d, f, k)) == form and d > 256
    words, tiles = -(-d // 128), -(-f // 128)
    room = max(64 * E, 512) * d * 4                                          # of the workspace's last area
    assert first == (form != 0 and tiles >= 32 and S * words * tiles >= 3e6 and S * words * 4 <= room)
    g = torch.Generator(device="cuda").manual_seed(T + d)
    x, wgu, wd = mx8(T, d, g, 1.0, scatter=True), mx8(E * 2 * f, d, g, 0.05), mx8(E * d, f, g, 0.05)
    slots = torch.randperm(S, device="cuda", generator=g).int()
    cut = torch.randint(0, S + 1, (E - 1,), device="cuda", generator=g).sort().values
    if E > 20:                                                               # uneven, but every expert has rows
        cut = (torch.arange(1, E, device="cuda") * S // E) + torch.randint(-S // E // 2, S // E // 2, (E - 1,), device="cuda", generator=g)
    off = torch.cat([cut.new_zeros(1), cut, cut.new_full((1,), S)]).int()
    got = run(T, E, d, f, k, (*x, slots), off, wgu, wd)
    want = run(T, E, d, f, k, in_group_order(x, slots, k), off, wgu, wd)
    for a, b in zip(got[:3], want[:3]):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    # against 64 bits: bounds as in test_gpu_mx8.py (inside an instruction 2^-11 of the sum of magnitudes; H to e4m3, Y to bfloat16)
    o = off.cpu().numpy()
    acc, rng = 2.0 ** -11, np.random.default_rng(T)
    val = lambda q, s: O.from_mx8(q.cpu().numpy(), s.cpu().numpy())  # noqa: E731
    for e in {0, int(np.argmax(np.diff(o))), E - 1}:
        if o[e] == o[e + 1]:
            continue
        rows = np.unique(np.concatenate([rng.integers(o[e], o[e + 1], 24), [o[e], o[e + 1] - 1]]))
        t = torch.from_numpy(rows).cuda()
        tok = slots[t].long() // k
        xv = val(x[0][tok], x[1][:, tok].contiguous())
        w = val(wgu[0][2 * f * e:2 * f * (e + 1)], wgu[1][:, 2 * f * e:2 * f * (e + 1)].contiguous())
        ab, m = xv @ w.T, np.abs(xv) @ np.abs(w).T
        a, b = ab[:, :f], ab[:, f:]
        sg = np.exp(-np.logaddexp(0.0, -a))
        h_ref = a * sg * b
        da, db = acc * m[:, :f], acc * m[:, f:]
        mag = da * np.abs(b) * (sg * (1 + np.abs(a) * (1 - sg))) + db * np.abs(a) * sg
        # silu's slope changes over the error of a sum (its second derivative is at most 1/2, its slope 1.1); the exponential is off by
        # the rounding of its argument, and infinite from 88 on, where silu is below 2e-36
        mag += da ** 2 * (np.abs(b) + db) / 2 + 1.1 * da * db + (1e-6 + np.abs(a) * 2.0 ** -23) * np.abs(h_ref) + 2e-36 * np.abs(b)
        h = val(got[0][t], got[1][:, t].contiguous())
        sc = np.transpose(got[1][:, t].cpu().numpy(), (1, 0, 2)).reshape(len(rows), -1)[:, :f // 32].astype(int)
        ex = np.repeat(sc - 127, 32, axis=1)
        assert (np.abs(h - h_ref) <= np.maximum(2.0 ** -4 * (np.abs(h_ref) + mag), 2.0 ** (ex - 10.0)) + mag).all(), e
        w = val(wd[0][d * e:d * (e + 1)], wd[1][:, d * e:d * (e + 1)].contiguous())
        y, y_ref, ym = got[2][t].double().cpu().numpy(), h @ w.T, np.abs(h) @ np.abs(w).T
        assert (np.abs(y - y_ref) <= 2.0 ** -8 * np.abs(y_ref) + (1 + 2.0 ** -8) * acc * ym).all(), e
        # a sum may cancel, a row of them does not: half a step of bfloat16 and the sums' own error
        assert (np.linalg.norm(y - y_ref, axis=1) <= (2.0 ** -8 + acc) * np.linalg.norm(y_ref, axis=1)).all(), e
