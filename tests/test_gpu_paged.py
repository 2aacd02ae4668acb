"""Append, attention, trees and acceptance over a batch's pages, against 64 bits.  Needs a real MI355X.

Slots that no sequence owns hold NaN in every test: what is read past a sequence's end shows."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import paged_reference as P
from paged_reference import DEV, Case

F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}           # half a step, relative


def _B():
    import paper_2404_12022_amd.binding as B
    return B


def say(msg):
    print(msg, flush=True)


def check(got, want, bound, what):
    got = got.double().cpu()
    off = (got - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} out of bound, worst {float((off - bound)[bad].nan_to_num(1e9).max()):.3e} past it, " \
                          f"first at {bad.nonzero()[0].tolist()}: {float(got[bad][0])} for {float(want[bad][0])}"


def attend(case, Hq, trees=True, **kw):
    B = _B()
    pools = [p.to(DEV) for p in case.new_pools()]
    q = case.normal(case.rows, Hq, case.hd, sigma=1.5).to(DEV)
    batch = case.batch(B, pools)
    out = torch.full((case.rows, Hq, case.hd), 77.0, dtype=case.dtype, device=DEV)
    B.ht_paged_attention(batch, q, pools[0], pools[1], case.anc().to(DEV) if trees else None, out=out, **kw)
    torch.cuda.synchronize()
    want, weight, size = P.attention(case, q, pools[0], pools[1], scale=kw.get("scale"))
    check(out[:case.used], want, P.attention_bound(case, want, weight, size), "attention")
    assert (out[case.used:] == 77.0).all()
    return out


HEADS = [(4, 4, 64), (8, 1, 64), (6, 3, 128), (16, 2, 128)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("Hq,Hkv,hd", HEADS + [(2, 1, 2), (3, 3, 80), (2, 2, 256), (4, 2, 34)])
@pytest.mark.parametrize("page", [8, 16, 64])
def test_attention_of_trees_of_all_sizes(dtype, Hq, Hkv, hd, page):
    """Sequences from nothing cached to several tiles, from no row to a full pass, in one call; two rows of no sequence behind."""
    say(f"attention {dtype} heads {Hq}/{Hkv} x {hd}, pages of {page}")
    attend(Case([0, 1, 15, 16, 63, 64, 65, 130, 200, 7], [1, 0, 3, 16, 17, 1, 33, 5, 9, 64], Hkv, hd, page, dtype, 11, spare_rows=2), Hq)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("Hq,Hkv,hd", HEADS)
@pytest.mark.parametrize("rows", [1, 2, 16, 17, 63, 65, 128, 129, 256])
def test_attention_of_chains(dtype, Hq, Hkv, hd, rows):
    say(f"chain {dtype} heads {Hq}/{Hkv} x {hd}, {rows} rows")
    attend(Case([0, 100, 31], [rows, max(1, rows // 2), rows], Hkv, hd, 32, dtype, 12, trees=False), Hq, trees=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("Hq,Hkv,hd,rows", [(4, 4, 64, 1), (16, 2, 128, 1), (16, 2, 128, 5), (4, 4, 128, 40), (16, 2, 128, 33)])
@pytest.mark.parametrize("length", [511, 1024, 4097, 20000])
def test_attention_over_long_caches(dtype, Hq, Hkv, hd, rows, length):
    """Long axes are split and joined; one sequence beside it is short."""
    say(f"long {dtype} heads {Hq}/{Hkv} x {hd}, {rows} rows over {length}")
    attend(Case([length, 3], [rows, rows], Hkv, hd, 16, dtype, 13), Hq)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_counts_every_key_once(dtype):
    """Equal scores and values of one unit vector per key: the output counts the keys, to a 60th or better."""
    B = _B()
    for hd, rows in ((64, 1), (128, 1), (128, 20), (64, 40)):
        for n in (0, 1, 7, 8, 31, 32, 33, 63, 64):
            case = Case([n, n + 3], [rows, 1], 2, hd, 8, dtype, 14)
            k, v = case.new_pools()
            for b in range(2):
                S = case.lens[b] + case.counts[b]
                page, row = case.where(b, range(S))
                k[page, :, row] = 0
                x = torch.zeros(S, 2, hd, dtype=dtype)
                x[range(S), :, [j % hd for j in range(S)]] = 1
                v[page, :, row] = x
            k, v = k.to(DEV), v.to(DEV)
            q = case.normal(case.rows, 4, hd).to(DEV)
            out = B.ht_paged_attention(case.batch(B, (k, v)), q, k, v, case.anc().to(DEV)).double().cpu()
            for b in range(2):
                for r in range(case.counts[b]):
                    slots = list(range(case.lens[b])) + [case.lens[b] + u for u in case.lines[b][r]]
                    want = torch.zeros(hd, dtype=torch.float64)
                    for j in slots:
                        want[j % hd] += 1.0 / len(slots)
                    # the reciprocal, the product and the result's rounding
                    assert ((out[case.starts[b] + r] - want).abs() <= (2 ** -21 + HALF[dtype] * 1.01) * want).all(), (hd, rows, n, b, r)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hd,rows", [(64, 1), (128, 12), (128, 70)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_row_does_not_see_does_not_matter(dtype, hd, rows, bad):
    """Keys and values of a tree's other branches that are no numbers; rows that see nothing; bits of rows that are not there."""
    B = _B()
    case = Case([20, 0, 70], [rows, max(2, rows), rows], 2, hd, 16, dtype, 15)
    k, v = [p.to(DEV) for p in case.new_pools()]
    masks = torch.zeros(case.used, 256, dtype=torch.bool)
    for b in range(3):
        t, at = case.counts[b], case.starts[b]
        poisoned = t // 2 if t > 1 else None
        if poisoned is not None:
            page, row = case.where(b, [case.lens[b] + poisoned])
            k[page.to(DEV), :, row.to(DEV)] = bad
            v[page.to(DEV), :, row.to(DEV)] = bad
        for r in range(t):
            masks[at + r, [u for u in case.lines[b][r] if u != poisoned]] = True
            masks[at + r, t:] = True                                # bits past the last row
    masks[case.starts[1] + 1] = False                               # nothing cached, no bit: an empty row
    bits = torch.stack([P.mask_words([[u for u in range(256) if m[u]]])[0] for m in masks.tolist()])
    q = case.normal(case.rows, 6, hd).to(DEV)
    out = B.ht_paged_attention(case.batch(B, (k, v)), q, k, v, bits.to(DEV))
    want, weight, size = P.attention(case, q, k, v, masks=masks)
    assert torch.isfinite(want).all()
    check(out, want, P.attention_bound(case, want, weight, size), "masked rows")
    assert (out[case.starts[1] + 1] == 0).all()


def test_a_value_that_is_no_number_reaches_the_rows_that_see_it():
    B = _B()
    for dtype in (F32, BF16):
        for rows, hd in ((1, 64), (9, 128), (40, 128)):
            case = Case([30], [rows], 1, hd, 16, dtype, 16, trees=False)
            k, v = [p.to(DEV) for p in case.new_pools()]
            page, row = case.where(0, [5])
            v[page.to(DEV), :, row.to(DEV), 3] = float("nan")
            out = B.ht_paged_attention(case.batch(B, (k, v)), case.normal(rows, 2, hd).to(DEV), k, v)
            assert out[:, :, 3].isnan().all() and torch.isfinite(out[:, :, 4:]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_pages_that_are_none_are_seen_by_nobody(dtype):
    B = _B()
    for hd, rows in ((64, 1), (128, 24)):
        case = Case([150, 40], [rows, rows], 2, hd, 16, dtype, 17)
        pools = [p.to(DEV) for p in case.new_pools()]
        case.table[0, 2], case.table[0, 5], case.table[1, 0], case.table[0, 7] = -1, case.pool, -2 ** 31, 2 ** 31 - 1
        q = case.normal(case.rows, 4, hd).to(DEV)
        out = B.ht_paged_attention(case.batch(B, pools), q, *pools, case.anc().to(DEV))
        want, weight, size = P.attention(case, q, *pools)
        check(out, want, P.attention_bound(case, want, weight, size), "missing pages")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_tables_that_break_the_host_s_bounds(dtype):
    """Lengths and row counts past the bounds, row starts that fall back or leave the rows: held to the bounds."""
    B = _B()
    case = Case([40, 20, 30], [6, 4, 5], 2, 64, 16, dtype, 18)
    pools = [p.to(DEV) for p in case.new_pools()]
    q = case.normal(case.rows, 4, 64).to(DEV)
    anc = case.anc().to(DEV)
    plain = B.ht_paged_attention(case.batch(B, pools), q, *pools, anc)
    batch = case.batch(B, pools)
    batch.tensors[1][0] = 2 ** 31 - 1                               # max_len is 40: the same
    assert torch.equal(B.ht_paged_attention(batch, q, *pools, anc), plain)
    batch.tensors[1][0] = -5                                        # as 0
    first = B.ht_paged_attention(batch, q, *pools, anc)
    case.lens[0] = 0
    want, weight, size = P.attention(case, q, *pools)
    check(first, want, P.attention_bound(case, want, weight, size), "length below 0")
    case.lens[0] = 40
    batch = case.batch(B, pools)
    batch.tensors[0].copy_(torch.tensor([0, 6, 10, 2 ** 31 - 1]))   # the last sequence: up to the last row
    assert torch.equal(B.ht_paged_attention(batch, q, *pools, anc), plain)
    batch.tensors[0].copy_(torch.tensor([0, 6, 3, -2 ** 31]))       # two sequences without rows
    out = torch.full_like(q, 5.0)
    B.ht_paged_attention(batch, q, *pools, anc, out=out)
    assert torch.equal(out[:6], plain[:6]) and (out[6:] == 5.0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_strides_scale_and_heads_apart(dtype):
    B = _B()
    for rows, hd in ((1, 64), (20, 128)):
        case = Case([33, 80], [rows, rows], 2, hd, 32, dtype, 19)
        pools = [p.to(DEV) for p in case.new_pools()]
        wide = case.normal(case.rows, 11, hd).to(DEV)
        q, out = wide[:, 3:7], torch.zeros(case.rows, 9, hd, dtype=dtype, device=DEV)
        B.ht_paged_attention(case.batch(B, pools), q, *pools, case.anc().to(DEV), scale=0.3, out=out[:, 1:5])
        want, weight, size = P.attention(case, q, *pools, scale=0.3)
        check(out[:, 1:5], want, P.attention_bound(case, want, weight, size), "strided")
        assert (out[:, 0] == 0).all() and (out[:, 5:] == 0).all()
        # rows that do not lie on 16 bytes
        raw = torch.zeros(q.numel() + 1, dtype=dtype, device=DEV)
        raw[1:] = q.reshape(-1)
        got = B.ht_paged_attention(case.batch(B, pools), raw[1:].view(q.shape), *pools, case.anc().to(DEV), scale=0.3)
        check(got, want, P.attention_bound(case, want, weight, size), "odd addresses")


def test_attention_over_a_pool_of_more_than_2_31_elements():
    B = _B()
    page, Hkv, hd = 64, 8, 128
    pool = 2 ** 31 // (page * Hkv * hd) + 40
    case = Case([300, 65], [1, 20], Hkv, hd, page, BF16, 20, last_pages=True, pool=pool)
    small = Case([300, 65], [1, 20], Hkv, hd, page, BF16, 20)
    case.parents, case.lines = small.parents, small.lines             # the same trees
    k, v = small.new_pools()
    pools = [torch.empty(pool, Hkv, page, hd, dtype=BF16, device=DEV) for _ in range(2)]
    for big, x in zip(pools, (k, v)):
        for b in range(2):
            w = -(-(small.lens[b] + small.counts[b]) // page)
            big[case.table[b, :w].long().to(DEV)] = x[small.table[b, :w].long()].to(DEV)
    assert int(case.table.max()) * page * Hkv * hd > 2 ** 31 - 2 ** 22
    q = case.normal(case.rows, 16, hd).to(DEV)
    out = B.ht_paged_attention(case.batch(B, pools), q, *pools, case.anc().to(DEV))
    want, weight, size = P.attention(small, q, k, v)
    check(out, want, P.attention_bound(small, want, weight, size), "far pages")


# ------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("Hq,Hkv,hd,rot", [(4, 4, 64, 64), (8, 1, 128, 128), (6, 3, 128, 64), (3, 1, 80, 34), (2, 2, 256, 256),
                                           (2, 1, 2, 2), (5, 5, 64, 0), (40, 8, 128, 34), (4, 2, 96, 48)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm,scaled", [(False, False), (True, True), (True, False)])
def test_append(dtype, Hq, Hkv, hd, rot, interleaved, norm, scaled):
    B = _B()
    say(f"append {dtype} heads {Hq}/{Hkv} x {hd}, {rot} turn, interleaved {interleaved} norm {norm} scaled {scaled}")
    case = Case([0, 15, 100, 7, 40000], [3, 0, 18, 33, 1], Hkv, hd, 16, dtype, 21, spare_rows=2)
    pools = [p.to(DEV) for p in case.new_pools()]
    before = [p.clone() for p in pools]
    fused = case.normal(case.rows, Hq + 2 * Hkv, hd).to(DEV)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    gains = [case.normal(hd, sigma=0.2, mean=1.0).to(DEV) if norm else None for _ in range(2)]
    freq = 10000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / max(rot, 1))
    inv = (freq / (1 + torch.arange(rot // 2) % 3)).float() if scaled else None
    amp = 1.2079441 if scaled else 1.0
    amp = float(torch.tensor(amp, dtype=F32))
    depth = case.depth()
    out = torch.full_like(q, 9.0)
    B.ht_paged_append(case.batch(B, pools), q, k, v, *pools, depth=depth.to(DEV), q_gain=gains[0], k_gain=gains[1], eps=1e-5, rot=rot,
                      interleaved=interleaved, inv_freq=None if inv is None else inv.to(DEV), amplitude=amp, q_out=out)
    pos = torch.tensor([case.lens[b] for b in range(case.seqs) for _ in range(case.counts[b])] + [0] * 2) + depth
    eps = float(torch.tensor(1e-5, dtype=F32))
    want = [P.turned(x, g, eps, pos, rot, interleaved, freq if inv is None else inv, amp) for x, g in ((q, gains[0]), (k, gains[1]))]
    # the factor rounded (twice with an amplitude), two products and a sum, and the norm: a sum of hd squares, root, quotient, gain
    slack = (8 + (hd / 2 + 8 if norm else 0)) * 2.0 ** -24
    half = HALF[dtype]
    n = case.used
    check(out[:n], want[0][0][:n], want[0][0][:n].abs() * half + (1 + half) * slack * want[0][1][:n] + 1e-38, "q")
    assert (out[n:] == 9.0).all()
    expect = [p.clone() for p in before]
    for b in range(case.seqs):
        at, t = case.starts[b], case.counts[b]
        if not t:
            continue
        page, row = (x.to(DEV) for x in case.where(b, range(case.lens[b], case.lens[b] + t)))
        got = pools[0][page, :, row]
        w, s = (x[at:at + t] for x in want[1])
        check(got, w, w.abs() * half + (1 + half) * slack * s + 1e-38, f"keys of sequence {b}")
        expect[0][page, :, row] = got
        expect[1][page, :, row] = v[at:at + t]
    for got, e in zip(pools, expect):                               # nothing else moved (NaN counts as itself)
        assert torch.equal(got.view(torch.int16 if dtype == BF16 else torch.int32), e.view(torch.int16 if dtype == BF16 else torch.int32))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_append_of_parts_in_place_and_without_pages(dtype):
    B = _B()
    case = Case([5, 30], [4, 9], 2, 64, 16, dtype, 22)
    pools = [p.to(DEV) for p in case.new_pools()]
    q, k, v = (case.normal(case.rows, h, 64).to(DEV) for h in (4, 2, 2))
    whole = [p.clone() for p in pools]
    out = B.ht_paged_append(case.batch(B, pools), q, k, v, *whole, rot=32)
    only = [p.clone() for p in pools]
    assert B.ht_paged_append(case.batch(B, pools), None, k, v, *only, rot=32) is None
    for a, b in zip(whole, only):
        assert torch.equal(a.nan_to_num(7), b.nan_to_num(7))
    assert torch.equal(B.ht_paged_append(case.batch(B, pools), q, None, None, None, None, rot=32), out)
    mine = q.clone()
    B.ht_paged_append(case.batch(B, pools), mine, None, None, None, None, rot=32, q_out=mine)
    assert torch.equal(mine, out)
    # odd addresses
    raw = torch.zeros(q.numel() + 1, dtype=dtype, device=DEV)
    raw[1:] = q.reshape(-1)
    assert torch.equal(B.ht_paged_append(case.batch(B, pools), raw[1:].view(q.shape), None, None, None, None, rot=32), out)
    # a page that is none: its rows are left out, the others stored
    case.table[1, 2] = case.pool + 3                                # slots 32 to 47 of the second sequence
    part = [p.clone() for p in pools]
    B.ht_paged_append(case.batch(B, pools), q, k, v, *part, rot=32)
    page, row = (x.to(DEV) for x in case.where(1, [30, 31]))
    assert torch.equal(part[1][page, :, row], v[4:6])
    touched = sum(int((a.nan_to_num(7) != b.nan_to_num(7)).any(-1).any(1).sum()) for a, b in zip(part, pools))
    assert touched == 2 * (4 + 2)


def test_append_at_far_positions():
    """Angles of hundreds of thousands of radians."""
    B = _B()
    case = Case([1000003], [2], 1, 64, 4096, F32, 23)
    pools = [torch.zeros(case.pool, 1, 4096, 64, device=DEV) for _ in range(2)]
    q = torch.ones(2, 1, 64, device=DEV)
    inv = torch.tensor([1.0 / (1 + j) for j in range(32)], dtype=F32)
    for freq in (None, inv):
        out = B.ht_paged_append(case.batch(B, pools), q, None, None, None, None, inv_freq=None if freq is None else freq.to(DEV))
        f = 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32) if freq is None else freq
        want, size = P.turned(q, None, 0.0, torch.tensor([1000003, 1000004]), 64, False, f, 1.0)
        # 10000^(-j/32) itself is given to 2^-53 by the reference: times a million, 1e-10
        check(out, want, 8 * 2.0 ** -24 * size + 1e-9, "far positions")


# ------------------------------------------------------------------------------------------------ trees, acceptance
def test_tree_tables():
    B = _B()
    case = Case([0, 5, 9, 1], [256, 0, 1, 70], 1, 64, 16, BF16, 24, spare_rows=3)
    pools = [p.to(DEV) for p in case.new_pools()]
    depth, anc = B.ht_tree_tables(case.batch(B, pools), case.flat_parents().to(DEV))
    assert torch.equal(depth[:case.used].cpu(), case.depth()[:case.used]) and torch.equal(anc[:case.used].cpu(), case.anc()[:case.used])
    # a parent that is not an earlier row: a root
    flat = case.flat_parents()
    flat[10], flat[20], flat[30] = 10, 255, -7
    depth, anc = B.ht_tree_tables(case.batch(B, pools), flat.to(DEV))
    for v in (10, 20, 30):
        assert int(depth[v]) == 0 and anc[v].tolist() == P.mask_words([[v]])[0].tolist()


def _answers(case, follow=0.85):
    tok = torch.randint(50, (case.rows,), generator=case.g, dtype=torch.int32)
    ans = torch.randint(50, (case.rows,), generator=case.g, dtype=torch.int32)
    for b in range(case.seqs):
        at = case.starts[b]
        for v in range(case.counts[b]):
            kids = [u for u in range(v + 1, case.counts[b]) if case.parents[b][u] == v]
            if kids and float(torch.rand((), generator=case.g)) < follow:
                ans[at + v] = tok[at + kids[int(torch.randint(len(kids), (), generator=case.g))]]
    return tok, ans


@pytest.mark.parametrize("dtype,hd,Hkv", [(F32, 64, 4), (BF16, 128, 8), (BF16, 2, 1), (F32, 34, 3), (BF16, 80, 1)])
@pytest.mark.parametrize("layers,max_path", [(1, 4), (3, 16), (2, 256)])
def test_acceptance(dtype, hd, Hkv, layers, max_path):
    B = _B()
    say(f"accept {dtype} {Hkv} x {hd}, {layers} layers, paths to {max_path}")
    case = Case([0, 15, 33, 8, 100, 3], [1, 8, 64, 0, 256, 130], Hkv, hd, 16, dtype, 25 + layers, layers=layers, spare_rows=2)
    pools = [p.to(DEV) for p in case.new_pools()]
    tok, ans = _answers(case)
    before = [p.cpu().clone() for p in pools]
    got = B.ht_paged_accept(case.batch(B, pools), *pools, case.flat_parents().to(DEV), tok.to(DEV), ans.to(DEV), max_path)
    n, path, emitted, root, length = (x.cpu() for x in got)
    longest = 0
    for b in range(case.seqs):
        t, at = case.counts[b], case.starts[b]
        if not t:
            assert int(n[b]) == 0 and int(root[b]) == -1 and int(length[b]) == case.lens[b] and (path[b] == -1).all()
            continue
        want = P.accept(case.parents[b], tok[at:at + t].tolist(), ans[at:at + t].tolist(), max_path)
        longest = max(longest, len(want))
        assert int(n[b]) == len(want) and int(length[b]) == case.lens[b] + len(want)
        assert path[b].tolist() == want + [-1] * (max_path - len(want))
        assert emitted[b].tolist() == [int(tok[at + v]) for v in want] + [-1] * (max_path - len(want))
        assert int(root[b]) == int(ans[at + want[-1]])
        for j, v in enumerate(want):
            (ps, rs), (pd, rd) = case.where(b, [case.lens[b] + v]), case.where(b, [case.lens[b] + j])
            for pool in before:
                pool[:, pd, :, rd] = pool[:, ps, :, rs].clone()
    assert longest >= 3
    for pool, want in zip(pools, before):
        as_int = torch.int16 if dtype == BF16 else torch.int32
        assert torch.equal(pool.cpu().view(as_int), want.view(as_int))


def test_acceptance_takes_the_first_of_equal_children_and_whole_chains():
    B = _B()
    case = Case([4, 0], [6, 256], 1, 64, 16, F32, 26, trees=False)
    case.parents[0] = [-1, 0, 0, 0, 2, 2]
    pools = [p.to(DEV) for p in case.new_pools()]
    tok = torch.cat([torch.tensor([9, 5, 7, 7, 3, 3]), torch.arange(256)]).int()
    ans = torch.cat([torch.tensor([7, 1, 3, 2, 8, 6]), torch.arange(1, 257)]).int()
    n, path, emitted, root, length = B.ht_paged_accept(case.batch(B, pools), *pools, case.flat_parents().to(DEV), tok.to(DEV), ans.to(DEV), 256)
    assert path[0, :3].tolist() == [0, 2, 4] and int(root[0]) == 8 and n.tolist() == [3, 256]
    assert path[1].tolist() == list(range(256)) and int(root[1]) == 256 and length.tolist() == [7, 256]


def test_shared_prompt_pages_stay_as_they_are():
    """Two continuations of one prompt: the same pages in front, pages of their own behind."""
    B = _B()
    case = Case([64, 64], [20, 20], 2, 64, 16, BF16, 27)
    case.table[1, :4] = case.table[0, :4]
    pools = [p.to(DEV) for p in case.new_pools()]
    shared = [p[case.table[0, :4].long().to(DEV)].clone() for p in pools]
    q, k, v = (case.normal(case.rows, h, 64).to(DEV) for h in (4, 2, 2))
    batch = case.batch(B, pools)
    depth, anc = B.ht_tree_tables(batch, case.flat_parents().to(DEV))
    assert torch.equal(depth.cpu(), case.depth()) and torch.equal(anc.cpu(), case.anc())
    qr = B.ht_paged_append(batch, q, k, v, *pools, depth=depth)
    out = B.ht_paged_attention(batch, qr, *pools, anc)
    want, weight, size = P.attention(case, qr, *pools)
    check(out, want, P.attention_bound(case, want, weight, size), "forked")
    tok, ans = _answers(case)
    B.ht_paged_accept(batch, *pools, case.flat_parents().to(DEV), tok.to(DEV), ans.to(DEV), 20)
    for p, s in zip(pools, shared):
        assert torch.equal(p[case.table[0, :4].long().to(DEV)], s)


# ------------------------------------------------------------------------------------------------ together
def _step(B, case, batch, pools, w, x, parent, tok, u, layers, Hq, hd, Hkv):
    """A verify step of a model without feed-forward blocks: tables, append and attention per layer, logits, sample, accept."""
    depth, anc = B.ht_tree_tables(batch, parent)
    for l in range(layers):
        y = (x @ w["qkv"][l]).view(-1, Hq + 2 * Hkv, hd)
        q = B.ht_paged_append(batch, y[:, :Hq], y[:, Hq:Hq + Hkv], y[:, Hq + Hkv:], pools[0][l], pools[1][l], depth=depth,
                              q_gain=w["gain"], k_gain=w["gain"], eps=1e-5, rot=hd // 2, interleaved=True)
        x = x + B.ht_paged_attention(batch, q, pools[0][l], pools[1][l], anc).flatten(1) @ w["o"][l]
    z = x @ w["head"]
    answers, _ = B.ht_sample_rows(z, u, torch.full_like(u, 0.8), None, torch.full_like(u, 0.9))
    return z, answers, B.ht_paged_accept(batch, *pools, parent, tok, answers, 8)


def _plain_step(case, pools, w, x, tok, u, layers, Hq, hd, Hkv):
    pos = torch.tensor([case.lens[b] for b in range(case.seqs) for _ in range(case.counts[b])]) + case.depth()
    freq = 10000.0 ** (-2.0 * torch.arange(hd // 4, dtype=torch.float64) / (hd // 2))
    for l in range(layers):
        y = (x @ w["qkv"][l].double().cpu()).view(-1, Hq + 2 * Hkv, hd)
        eps = float(torch.tensor(1e-5, dtype=F32))
        q, k = (P.turned(t, w["gain"], eps, pos, hd // 2, True, freq, 1.0)[0] for t in (y[:, :Hq], y[:, Hq:Hq + Hkv]))
        for b in range(case.seqs):
            at, t = case.starts[b], case.counts[b]
            page, row = case.where(b, range(case.lens[b], case.lens[b] + t))
            pools[0][l][page, :, row] = k[at:at + t]
            pools[1][l][page, :, row] = y[at:at + t, Hq + Hkv:]
        x = x + P.attention(case, q, pools[0][l], pools[1][l])[0].flatten(1) @ w["o"][l].double().cpu()
    z = x @ w["head"].double().cpu()
    drawn = [P.sample(z[r].numpy(), float(u[r]), float(torch.tensor(0.8)), 0, float(torch.tensor(0.9))) for r in range(case.used)]
    return z, drawn


@pytest.mark.parametrize("captured", [False, True])
def test_verify_steps_of_a_batch(captured):
    """Three steps of three sequences, float32, eager and as one captured graph that is replayed with new contents; the caches carry
    over.  After every step the logits, the sampled tokens (away from borders), the accepted paths and the caches are compared."""
    B = _B()
    Hq, Hkv, hd, layers, V, d = 4, 2, 64, 2, 300, 96
    case = Case([17, 3, 40], [12, 7, 9], Hkv, hd, 16, F32, 30, layers=layers)
    case.max_len = 100
    g = case.g
    width = -(-(case.max_len + case.max_rows) // 16)
    table = torch.randperm(3 * width, generator=g).int().view(3, width)     # room for all steps
    old, case.table, case.pool = case.table, table, 3 * width
    plain = [torch.zeros(layers, case.pool, Hkv, 16, hd, dtype=torch.float64) for _ in range(2)]
    for b in range(3):
        page, row = case.where(b, range(case.lens[b]))
        for p in plain:
            p[:, page, :, row] = torch.randn(case.lens[b], layers, Hkv, hd, generator=g).double()
    pools = [p.float().to(DEV) for p in plain]
    plain = [p.double().cpu() for p in pools]
    w = {"qkv": [torch.randn(d, (Hq + 2 * Hkv) * hd, generator=g).mul(d ** -0.5).to(DEV) for _ in range(layers)],
         "o": [torch.randn(Hq * hd, d, generator=g).mul((Hq * hd) ** -0.5).to(DEV) for _ in range(layers)],
         "head": torch.randn(d, V, generator=g).mul(3 * d ** -0.5).to(DEV), "gain": torch.rand(hd, generator=g).add(0.5).to(DEV)}
    emb = torch.randn(V, d, generator=g).to(DEV)
    batch = case.batch(B, pools)
    length = batch.tensors[1]
    tok_d, u_d = torch.zeros(case.used, dtype=torch.int32, device=DEV), torch.zeros(case.used, device=DEV)
    parent_d, x_d = torch.zeros(case.used, dtype=torch.int32, device=DEV), torch.zeros(case.used, d, device=DEV)
    run = lambda: _step(B, case, batch, pools, w, x_d, parent_d, tok_d, u_d, layers, Hq, hd, Hkv)  # noqa: E731
    graph = None
    moved = 0
    for step in range(3):
        case.parents = [P.random_parents(t, g) for t in case.counts]
        case.lines = [P.lines_of(p) for p in case.parents]
        # drafted tokens: what the model would answer, for most rows, so that paths are accepted
        tok = torch.randint(V, (case.used,), generator=g, dtype=torch.int32)
        u = torch.rand(case.used, generator=g)
        for _ in range(2):
            z, drawn = _plain_step(case, [p.clone() for p in plain], w, emb.cpu().double()[tok.long()], tok, u, layers, Hq, hd, Hkv)
            for b in range(3):
                for v in range(1, case.counts[b]):
                    if case.parents[b][v] == v - 1 or v % 2:
                        tok[case.starts[b] + v] = drawn[case.starts[b] + case.parents[b][v]][0]
        z, drawn = _plain_step(case, plain, w, emb.cpu().double()[tok.long()], tok, u, layers, Hq, hd, Hkv)
        tok_d.copy_(tok), u_d.copy_(u), parent_d.copy_(case.flat_parents()), x_d.copy_(emb[tok.long().to(DEV)])
        if captured and graph is None:
            # (what a capture's warm-up and capture leave in the pages are this step's rows: the replay stores them again)
            saved = [p.clone() for p in pools]
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                run()
            torch.cuda.current_stream().wait_stream(side)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                result = run()
            for p, s in zip(pools, saved):
                p.copy_(s)
        if captured:
            graph.replay()
        else:
            result = run()
        torch.cuda.synchronize()
        zg, answers, (n, path, emitted, root, new_len) = result
        # logits of order 3 through two layers of float32: products of 96 and 256 terms, 1e-4 is a hundred times their roundings
        assert (zg.double().cpu() - z).abs().max() < 1e-4
        for r, (t, _, near) in enumerate(drawn):
            assert near < 1e-4 or int(answers[r]) == t
        for b in range(3):
            at, t = case.starts[b], case.counts[b]
            want = P.accept(case.parents[b], tok[at:at + t].tolist(), answers[at:at + t].tolist(), 8)
            assert path[b, :len(want)].tolist() == want and int(n[b]) == len(want)
            moved += sum(v != j for j, v in enumerate(want))
            for j, v in enumerate(want):
                (ps, rs), (pd, rd) = case.where(b, [case.lens[b] + v]), case.where(b, [case.lens[b] + j])
                for p in plain:
                    p[:, pd, :, rd] = p[:, ps, :, rs].clone()
            case.lens[b] += len(want)
            page, row = case.where(b, range(case.lens[b]))
            for p, q in zip(pools, plain):
                assert (p.double().cpu()[:, page, :, row] - q[:, page, :, row]).abs().max() < 1e-4
        assert new_len.tolist() == case.lens
        length.copy_(new_len)
    assert moved >= 3


def test_attention_in_two_captured_graphs_beside_eager_calls():
    """Every graph with its scratch; each replayed several times between eager calls over other contents."""
    B = _B()
    case = Case([3000, 50], [4, 4], 2, 128, 16, BF16, 31)
    pools = [p.to(DEV) for p in case.new_pools()]
    qs = [case.normal(case.rows, 16, 128).to(DEV) for _ in range(3)]
    batch, anc = case.batch(B, pools), case.anc().to(DEV)
    want = [B.ht_paged_attention(batch, q, *pools, anc) for q in qs]
    graphs = []
    for q in qs[:2]:
        scratch, out = B.ht_paged_attention_scratch(batch, 16), torch.zeros_like(q)
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            B.ht_paged_attention(batch, q, *pools, anc, out=out, scratch=scratch)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.ht_paged_attention(batch, q, *pools, anc, out=out, scratch=scratch)
        graphs.append((graph, out, scratch))
    for _ in range(3):
        for i, (graph, out, _s) in enumerate(graphs):
            out.zero_()
            graph.replay()
            assert torch.equal(B.ht_paged_attention(batch, qs[2], *pools, anc), want[2])
            torch.cuda.synchronize()
            assert torch.equal(out, want[i])


def test_calls_on_a_stream_of_their_own():
    B = _B()
    case = Case([900, 50], [4, 4], 2, 128, 16, BF16, 32)
    pools = [p.to(DEV) for p in case.new_pools()]
    q, k, v = (case.normal(case.rows, h, 128).to(DEV) for h in (16, 2, 2))
    batch, anc = case.batch(B, pools), case.anc().to(DEV)
    other = [p.clone() for p in pools]
    want = B.ht_paged_attention(batch, B.ht_paged_append(batch, q, k, v, *pools), *pools, anc)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    qr = B.ht_paged_append(batch, q, k, v, *other, stream=side)
    got = B.ht_paged_attention(batch, qr, *other, anc, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(other[0].nan_to_num(3), pools[0].nan_to_num(3))
