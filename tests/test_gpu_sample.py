"""Sampling from given numbers against 64 bits.  Needs a real MI355X.

Tokens have to be equal unless the number lies within 1e-12 of a border of the running sums (relative to their total), where the order
of 64-bit additions decides; no case is allowed more than a few of those.  Log shares: 64 bits rounded once, 2^-24 relative, and the
error of the sums, 1e-12."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paged_reference as P
from paged_reference import DEV

F32, BF16 = torch.float32, torch.bfloat16


def _B():
    import paper_2404_12022_amd.binding as B
    return B


def check(z, u, T=None, k=None, p=None, mp=None):
    B = _B()
    rows = z.shape[0]
    give = [None if x is None else torch.as_tensor(x).to(DEV) for x in (T, k, p, mp)]
    tokens, logprob = B.ht_sample_rows(z.to(DEV), u.to(DEV), *give)
    tokens, logprob = tokens.cpu(), logprob.double().cpu()
    zh = z.double().numpy()
    near_border = 0
    for r in range(rows):
        one = [d if x is None else float(x[r]) for x, d in ((T, 1.0), (k, 0), (p, 1.0), (mp, 0.0))]
        want, lp, near = P.sample(zh[r], float(u[r]), one[0], int(one[1]), one[2], one[3])
        if near < 1e-12:
            near_border += 1
            continue
        assert int(tokens[r]) == want, f"row {r}: {int(tokens[r])} for {want}, settings {one}, u {float(u[r])}, nearest border {near}"
        assert float(logprob[r]) == lp or abs(float(logprob[r]) - lp) <= 2 ** -24 * abs(lp) + 1e-12, (r, float(logprob[r]), lp)
    assert near_border <= max(1, rows // 50)


def _logits(rows, V, dtype, g, sigma=2.0):
    z = torch.randn(rows, V, generator=g) * sigma
    z += (torch.rand(rows, V, generator=g) < 40 / V) * torch.rand(rows, V, generator=g) * 9
    return z.to(dtype)


def _settings(rows, g):
    pick = lambda v, t: torch.tensor(v, dtype=t)[torch.randint(len(v), (rows,), generator=g)]  # noqa: E731
    return (pick([1.0, 0.7, 1.3, 0.05, 0.0, 5.0], F32), pick([0, 1, 2, 40, 999, 100000], torch.int32),
            pick([1.0, 0.9, 0.5, 0.999, 0.0], F32), pick([0.0, 0.05, 0.3, 1.0], F32))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 1000, 4095, 4096, 4097, 8193, 32000, 32768, 32769, 50257, 128001])
def test_all_filters_at_all_widths(dtype, V):
    g = torch.Generator().manual_seed(V)
    rows = 64 if V < 40000 else 24
    print(f"sample {dtype} V={V}", flush=True)
    z, u = _logits(rows, V, dtype, g), torch.rand(rows, generator=g)
    T, k, p, mp = _settings(rows, g)
    check(z, u, T, k, p, mp)
    check(z, u)
    check(z, u, T=T)
    check(z, u, k=k)
    check(z, u, p=p)
    check(z, u, mp=mp)
    check(z, u, T=T, p=p)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [300, 5000, 40001])
def test_rows_with_masks_infinities_and_nan(dtype, V):
    g = torch.Generator().manual_seed(5)
    z = _logits(24, V, dtype, g)
    lowest = torch.finfo(dtype).min
    hide = torch.rand(V, generator=g) < 0.6
    hide[7] = False
    for r, v in enumerate((-math.inf, lowest, math.nan, -1e30)):
        for i in range(4):
            z[4 * r + i, hide] = v
    z[16] = -math.inf                          # nothing left
    z[17] = math.nan
    z[18] = lowest
    z[19, [3, 50, 200]] = math.inf
    z[20] = -math.inf
    z[20, 250] = -5.0                          # one left
    z[21, ::2] = torch.finfo(dtype).max
    z[22] = 0.0
    z[22, ::3] = -0.0                          # equal values
    z[23] *= 1e30
    u = torch.rand(24, generator=g)
    for T, k, p, mp in ((1.0, 0, 1.0, 0.0), (0.7, 5, 1.0, 0.0), (1.2, 0, 0.6, 0.0), (1.0, 100, 0.8, 0.02), (0.0, 3, 0.5, 0.1),
                        (1.0, 20000, 0.95, 0.0)):
        full = lambda v, t: torch.full((24,), v, dtype=t)  # noqa: E731
        check(z, u, full(T, F32), full(k, torch.int32), full(p, F32), full(mp, F32))
    B = _B()
    tokens, lp = B.ht_sample_rows(z.to(DEV), u.to(DEV))
    assert tokens[16:18].tolist() == [-1, -1] and lp[16:18].tolist() == [-math.inf] * 2


@pytest.mark.parametrize("V", [2000, 30000, 70000])
def test_equal_values_go_by_index(V):
    """Many equal logits: the first ones by index are kept, more of them than a list holds."""
    g = torch.Generator().manual_seed(6)
    z = torch.zeros(12, V)
    z[6:] = torch.randint(0, 3, (6, V), generator=g).float()
    u = torch.rand(12, generator=g)
    u[0], u[6] = 0.999999, 0.999999
    for k in (1, 7, 1500, V - 1):
        check(z, u, k=torch.full((12,), k, dtype=torch.int32))
    # sums of equal halves, quarters and eighths are exact: the borders of the prefix are too
    for p in (0.25, 0.5, 0.125):
        check(z[:6], u[:6], p=torch.full((6,), p))
    check(z[6:], u[6:], k=torch.full((6,), 1900, dtype=torch.int32), p=torch.full((6,), 0.77))


def test_numbers_at_the_ends_and_odd_settings():
    g = torch.Generator().manual_seed(7)
    z = _logits(8, 700, F32, g)
    z[:, -1] = -math.inf
    u = torch.tensor([0.0, -1.0, math.nan, 1.0, 2.0, math.inf, 1 - 2 ** -24, 1e-30])
    check(z, u)
    check(z, u, k=torch.full((8,), 3, dtype=torch.int32))
    check(z, torch.rand(8, generator=g), T=torch.tensor([math.inf, math.nan, -1.0, 1e-30, 1e30, 1e-45, 2.0, 0.0]))
    check(z, torch.rand(8, generator=g), k=torch.tensor([-5, 0, 1, 699, 700, 701, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32),
          p=torch.tensor([math.nan, -1.0, 2.0, 0.5, 1e-30, 1 - 2 ** -24, 1.0, 0.3]),
          mp=torch.tensor([math.nan, -1.0, 2.0, 1.0, 1e-30, 0.5, 0.0, math.inf]))


def test_scales_far_apart():
    """Values over many orders of magnitude: the search's steps hold too many at first."""
    g = torch.Generator().manual_seed(8)
    z = -torch.exp(torch.rand(6, 20000, generator=g) * 60 - 30)
    u = torch.rand(6, generator=g)
    for k in (1, 30, 5000, 19999):
        check(z, u, k=torch.full((6,), k, dtype=torch.int32))
    check(z, u, T=torch.full((6,), 0.01), p=torch.full((6,), 0.7))
    check(z, u, T=torch.full((6,), 1e6), p=torch.full((6,), 0.37))


def test_strided_rows_chosen_outputs_streams_and_replays():
    B = _B()
    g = torch.Generator().manual_seed(9)
    wide = _logits(16, 5003, BF16, g).to(DEV)
    u = torch.rand(16, generator=g).to(DEV)
    for part in (wide[:, 1:4002], wide[::2, 3:], wide[:1, 5:]):
        rows = part.shape[0]
        tokens, lp = B.ht_sample_rows(part, u[:rows].contiguous())
        same, lp2 = B.ht_sample_rows(part.contiguous(), u[:rows].contiguous())
        assert torch.equal(tokens, same) and torch.equal(lp, lp2)
    tokens, lp = torch.full((16,), 9, dtype=torch.int32, device=DEV), torch.zeros(16, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = B.ht_sample_rows(wide, u, tokens=tokens, logprob=lp, stream=side)
    side.synchronize()
    want = B.ht_sample_rows(wide, u)
    assert out[0] is tokens and torch.equal(tokens, want[0]) and torch.equal(lp, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.ht_sample_rows(wide, u, tokens=tokens, logprob=lp)
    for i in range(4):
        u.copy_(torch.rand(16, generator=g))
        graph.replay()
        want = B.ht_sample_rows(wide, u)
        torch.cuda.synchronize()
        assert torch.equal(tokens, want[0]) and torch.equal(lp, want[1]), i


def test_shares_of_drawn_tokens():
    """Evenly spaced numbers draw every token as often as its share says, to one draw."""
    B = _B()
    g = torch.Generator().manual_seed(10)
    n = 4096
    z = torch.randn(1, 50, generator=g)
    tokens, _ = B.ht_sample_rows(z.expand(n, 50).contiguous().to(DEV), ((torch.arange(n) + 0.5) / n).to(DEV))
    count = np.bincount(tokens.cpu().numpy(), minlength=50)
    share = torch.softmax(z[0].double(), 0).numpy() * n
    assert np.abs(count - share).max() <= 1.0
    assert (tokens.cpu()[1:] >= tokens.cpu()[:-1]).all()
