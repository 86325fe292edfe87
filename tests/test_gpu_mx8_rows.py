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
