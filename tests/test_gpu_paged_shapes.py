"""Attention over pages where the work is cut differently: many sequences, many items, long ones in many parts, large groups, loose
bounds, and the calls that the interface allows besides (a result in place, odd layer strides, replays over other lengths).  Needs a real
MI355X.  The bounds are those of paged_reference.attention_bound."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import paged_reference as P
from paged_reference import DEV, Case

F32, BF16 = torch.float32, torch.bfloat16


def _B():
    import paper_2404_12022_amd.binding as B
    return B


def plain(case, q, pools, scale=None):
    """paged_reference.attention with a product for every sequence and key/value head."""
    Hq, hd = q.shape[1], q.shape[2]
    G, scale = Hq // case.Hkv, 1.0 / math.sqrt(hd) if scale is None else scale
    out = torch.zeros(case.used, Hq, hd, dtype=torch.float64)
    weight, size = torch.zeros_like(out), torch.zeros(case.used, Hq, 1, dtype=torch.float64)
    pools, qd = [p.cpu() for p in pools], q.double().cpu()
    for b in range(case.seqs):
        n, t, at = case.lens[b], case.counts[b], case.starts[b]
        if not t:
            continue
        (k, ok), (v, _) = case.slots(pools[0], b), case.slots(pools[1], b)
        seen = torch.zeros(t, n + t, dtype=torch.bool)
        seen[:, :n] = True
        for r in range(t):
            seen[r, [n + u for u in case.lines[b][r]]] = True
        seen = (seen & ok).repeat_interleave(G, 0)
        k, v = k.masked_fill(~ok[:, None, None], 0.0), v.masked_fill(~ok[:, None, None], 0.0)
        for h in range(case.Hkv):
            qh = qd[at:at + t, h * G:(h + 1) * G].reshape(t * G, hd)
            z = (qh @ k[:, h].T * scale).masked_fill(~seen, -math.inf)
            p = torch.softmax(z, 1).nan_to_num(0.0)
            s = (qh.abs() @ k[:, h].abs().T * scale).masked_fill(~seen, 0.0).amax(1)
            put = lambda x, w: x[at:at + t, h * G:(h + 1) * G].copy_(w.view(t, G, -1))  # noqa: E731
            put(out, p @ v[:, h])
            put(weight, p @ v[:, h].abs())
            put(size, s)
    return out, weight, size


def check(case, got, q, pools, what):
    want, weight, size = plain(case, q, pools)
    got = got[:case.used].double().cpu()
    bound = P.attention_bound(case, want, weight, size)
    off = (got - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, first at {bad.nonzero()[0].tolist()}: {float(got[bad][0])} for {float(want[bad][0])}"


def attend(case, Hq, what, **bounds):
    B = _B()
    print(what, flush=True)
    pools = [p.to(DEV) for p in case.new_pools()]
    q = case.normal(case.rows, Hq, case.hd, sigma=1.5).to(DEV)
    out = torch.full((case.rows, Hq, case.hd), 77.0, dtype=case.dtype, device=DEV)
    B.ht_paged_attention(case.batch(B, pools, **bounds), q, *pools, case.anc().to(DEV), out=out)
    check(case, out, q, pools, what)
    assert (out[case.used:] == 77.0).all()
    return pools, q, out


@pytest.mark.parametrize("dtype,rows", [(F32, 9), (BF16, 3), (BF16, 7), (BF16, 12), (BF16, 30)])
@pytest.mark.parametrize("seqs,Hq,Hkv", [(255, 8, 2), (256, 4, 1), (257, 8, 2), (300, 5, 1), (130, 32, 8)])
def test_many_sequences(dtype, rows, seqs, Hq, Hkv):
    g = torch.Generator().manual_seed(seqs)
    lens = torch.randint(0, 90, (seqs,), generator=g).tolist()
    counts = torch.randint(0, rows + 1, (seqs,), generator=g).tolist()
    lens[5], counts[-1] = 700, rows
    attend(Case(lens, counts, Hkv, 64, 16, dtype, 40, spare_rows=1), Hq, f"{dtype} {seqs} sequences of {rows} rows, {Hq} / {Hkv} heads")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("Hq,Hkv,rows", [(40, 8, 20), (64, 8, 16), (64, 8, 33), (16, 1, 5), (71, 1, 3), (256, 1, 2), (96, 32, 30), (3, 3, 200), (33, 3, 12)])
def test_groups_of_all_sizes(dtype, Hq, Hkv, rows):
    attend(Case([400, 0, 77], [rows, rows, max(rows // 2, 1)], Hkv, 128, 32, dtype, 41), Hq, f"{dtype} {Hq} / {Hkv} heads, {rows} rows")


@pytest.mark.parametrize("dtype,rows", [(F32, 40), (BF16, 1), (BF16, 14), (BF16, 30), (BF16, 256)])
@pytest.mark.parametrize("hd,length", [(64, 30011), (128, 12289)])
def test_one_long_sequence_beside_short_ones(dtype, rows, hd, length):
    attend(Case([length, 3, 0, 200], [rows, 1, rows, 0], 1, hd, 64, dtype, 42), 2, f"{dtype} {rows} rows over {length} of {hd}")


@pytest.mark.parametrize("dtype,rows", [(F32, 20), (BF16, 4), (BF16, 12), (BF16, 25), (BF16, 100)])
def test_bounds_far_above_what_is_there(dtype, rows):
    case = Case([90, 1, 33, 0], [rows, 1, rows // 2, 1], 2, 128, 8, dtype, 43)
    wide = torch.full((4, 4200), -1, dtype=torch.int32)
    wide[:, :case.table.shape[1]] = case.table
    case.table = wide
    attend(case, 4, f"{dtype} {rows} rows, loose bounds", max_rows=256, max_len=30000)


@pytest.mark.parametrize("dtype,hd,rows", [(F32, 64, 20), (F32, 128, 20), (BF16, 128, 3), (BF16, 64, 7), (BF16, 128, 7), (BF16, 64, 14), (BF16, 128, 14),
                                           (BF16, 64, 90), (BF16, 128, 90)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_missing_pages_and_values_that_are_no_numbers(dtype, hd, rows, bad):
    """Pages of 8 that are none, in front, in the middle and among the rows of the pass; in the rows of the pass keys and values of
    rows that others do not see hold `bad`: the first row's line stays clean, and so does every row that does not see row 1."""
    B = _B()
    case = Case([900, 40, 0], [rows, rows, rows], 2, hd, 8, dtype, 44)
    print(f"missing pages {dtype} {hd} {rows} {bad}", flush=True)
    pools = case.new_pools()
    for b, pages in ((0, (0, 50, 51) + ((113,) if rows > 4 else ())), (1, (2, 5)), (2, (0,))):
        case.table[b, list(pages)] = torch.tensor([-1, case.pool, -7, 2 ** 31 - 1][:len(pages)], dtype=torch.int32)
    clean = [p.clone() for p in pools]
    for b in range(3):
        page, row = case.where(b, [case.lens[b] + 1])
        if 0 <= int(page) < case.pool:
            for p, c in zip(pools, clean):
                p[page, :, row] = bad
                c[page, :, row] = 0.0
    pools, clean = [p.to(DEV) for p in pools], [p.to(DEV) for p in clean]
    q = case.normal(case.rows, 8, hd, sigma=1.5).to(DEV)
    out = B.ht_paged_attention(case.batch(B, pools), q, *pools, case.anc().to(DEV))
    want, weight, size = plain(case, q, clean)
    bound = P.attention_bound(case, want, weight, size)
    seen = 0
    for b in range(3):
        page, _ = case.where(b, [case.lens[b] + 1])
        held = 0 <= int(page) < case.pool
        for r in range(rows):
            got, at = out[case.starts[b] + r].double().cpu(), case.starts[b] + r
            if held and 1 in case.lines[b][r]:
                seen += 1
                assert not got.isfinite().any()
            else:
                assert ((got - want[at]).abs() <= bound[at]).all(), (b, r)
    assert seen


@pytest.mark.parametrize("dtype,rows", [(F32, 20), (BF16, 4), (BF16, 12), (BF16, 25), (BF16, 100)])
def test_the_result_in_place_of_the_queries(dtype, rows):
    B = _B()
    case = Case([2900, 40, 0], [rows, rows, max(rows // 3, 1)], 2, 128, 16, dtype, 45)
    pools = [p.to(DEV) for p in case.new_pools()]
    q = case.normal(case.rows, 6, 128, sigma=1.5).to(DEV)
    batch, anc = case.batch(B, pools), case.anc().to(DEV)
    want = B.ht_paged_attention(batch, q, *pools, anc)
    check(case, want, q, pools, "apart")
    assert B.ht_paged_attention(batch, q, *pools, anc, out=q) is q and torch.equal(q, want)


@pytest.mark.parametrize("dtype,rows", [(F32, 16), (BF16, 2), (BF16, 6), (BF16, 12), (BF16, 64)])
def test_replays_over_other_lengths_and_trees(dtype, rows):
    """A captured call over new row starts, lengths, pages and masks: what an eager call of them gives, bit for bit, and right."""
    B = _B()
    cases = [Case(lens, counts, 2, 64, 16, dtype, 46 + i, pool=600) for i, (lens, counts) in enumerate(
        (([4000, 10, 300], [rows, rows, rows]), ([0, 5, 7], [1, 0, rows]), ([1500, 2000, 1], [rows, 1, rows]), ([4000, 4000, 0], [0, rows, rows])))]
    rows_all, width = 3 * rows, 4096 // 16 + 64
    start, length = torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    table = torch.full((3, width), -1, dtype=torch.int32, device=DEV)
    pools = [torch.zeros(600, 2, 16, 64, dtype=dtype, device=DEV) for _ in range(2)]
    q, anc = torch.zeros(rows_all, 8, 64, dtype=dtype, device=DEV), torch.zeros(rows_all, 4, dtype=torch.int64, device=DEV)
    out = torch.zeros_like(q)
    batch = B.PagedBatch(start, length, table, *pools, rows_all, rows, 4000)
    scratch, own = B.ht_paged_attention_scratch(batch, 8), B.ht_paged_attention_scratch(batch, 8)

    def fill(case):
        start.copy_(torch.tensor(case.starts, dtype=torch.int32))
        length.copy_(torch.tensor(case.lens, dtype=torch.int32))
        table.fill_(-1)
        table[:, :case.table.shape[1]] = case.table.to(DEV)
        fresh = case.new_pools()
        for p, x in zip(pools, fresh):
            p.copy_(x)
        q[:case.used] = case.normal(case.used, 8, 64, sigma=1.5).to(DEV)
        anc[:case.rows] = case.anc().to(DEV)
        return fresh

    fill(cases[0])
    B.ht_paged_attention(batch, q, *pools, anc, out=out, scratch=scratch)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.ht_paged_attention(batch, q, *pools, anc, out=out, scratch=scratch)
    for turn in (0, 1, 2, 3, 1, 0):
        fresh = fill(cases[turn])
        out.fill_(77.0)
        graph.replay()
        want = torch.full_like(out, 77.0)
        B.ht_paged_attention(batch, q, *pools, anc, out=want, scratch=own)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert (out[cases[turn].used:] == 77.0).all()
        check(cases[turn], out, q[:cases[turn].used], fresh, f"replay {turn}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("extra", [0, 1, 5, 64])
def test_acceptance_over_layers_that_lie_apart(dtype, extra):
    """Layers any number of elements apart: through the C entry, which takes the distance."""
    B = _B()
    layers, hd = 3, 64
    case = Case([5, 20], [12, 30], 2, hd, 16, dtype, 48)
    pool = case.pool * 2 * 16 * hd
    step = pool + extra
    raw = [case.normal(layers * step).to(DEV) for _ in range(2)]
    before = [r.cpu().clone() for r in raw]
    tok, ans = torch.arange(case.rows).int(), torch.full((case.rows,), -9, dtype=torch.int32)
    for parents, first in zip(case.parents, case.starts):           # every row is answered with its last child
        for v in range(1, len(parents)):
            ans[first + parents[v]] = tok[first + v]
    dev = [x.to(DEV) for x in (case.flat_parents(), tok, ans)]
    shape = [r[:pool].view(case.pool, 2, 16, hd) for r in raw]
    batch = case.batch(B, shape)
    out = torch.zeros(3 * 2 + 2 * 2 * 8, dtype=torch.int32, device=DEV)
    at = out.data_ptr()
    rc = B.lib.ht_paged_accept(batch.ref, layers, step, raw[0].data_ptr(), raw[1].data_ptr(), *(x.data_ptr() for x in dev), 8,
                               at, at + 24, at + 24 + 64, at + 8, at + 16, torch.cuda.current_stream().cuda_stream)
    assert rc == B.HT_OK
    torch.cuda.synchronize()
    moved = 0
    for b in range(2):
        t, first = case.counts[b], case.starts[b]
        path = P.accept(case.parents[b], tok[first:first + t].tolist(), ans[first:first + t].tolist(), 8)
        for j, v in enumerate(path):
            moved += j != v
            (ps, rs), (pd, rd) = case.where(b, [case.lens[b] + v]), case.where(b, [case.lens[b] + j])
            for r in before:
                for layer in range(layers):
                    x = r[layer * step:layer * step + pool].view(case.pool, 2, 16, hd)
                    x[pd, :, rd] = x[ps, :, rs].clone()
    assert moved
    for r, want in zip(raw, before):
        assert torch.equal(r.cpu(), want)


def test_the_largest_vocabulary_and_many_rows():
    B = _B()
    V = B.HT_MAX_SAMPLE_VOCAB
    g = torch.Generator().manual_seed(49)
    for dtype in (F32, BF16):
        z = (torch.randn(4, V, generator=g) * 3).to(dtype)
        u = torch.rand(4, generator=g)
        for settings in ({}, dict(top_k=torch.tensor([7, 900, 5000, 0]).int(), top_p=torch.tensor([0.9, 0.5, 0.99, 0.7]))):
            tokens, lp = B.ht_sample_rows(z.to(DEV), u.to(DEV), **{n: x.to(DEV) for n, x in settings.items()})
            for r in range(4):
                want, share, near = P.sample(z[r].double().numpy(), float(u[r]), 1.0, int(settings["top_k"][r]) if settings else 0,
                                             float(settings["top_p"][r]) if settings else 1.0)
                assert near < 1e-12 or int(tokens[r]) == want
                assert near < 1e-12 or abs(float(lp[r]) - share) <= 2 ** -24 * abs(share) + 1e-12
    rows = 1 << 20
    z = torch.randn(rows, 5, generator=g)
    tokens, lp = B.ht_sample_rows(z.to(DEV), torch.rand(rows, generator=g).to(DEV), top_k=torch.ones(rows, dtype=torch.int32, device=DEV))
    assert torch.equal(tokens.cpu().long(), z.argmax(1)) and (lp == 0).all()


@pytest.mark.parametrize("Hkv,seqs,rows", [(300, 1, 40), (700, 1, 20), (5, 3, 100), (48, 2, 70)])
def test_heads_that_do_not_divide_the_grid(Hkv, seqs, rows):
    attend(Case([1500, 600, 40][:seqs], [rows, 3, rows][:seqs], Hkv, 64, 64, BF16, 50), Hkv, f"{Hkv} heads, {rows} rows")


@pytest.mark.parametrize("dtype,rows,hd", [(F32, 20, 64), (BF16, 2, 128), (BF16, 12, 128), (BF16, 100, 64), (BF16, 5, 80)])
def test_a_batch_that_has_nothing_to_do(dtype, rows, hd):
    """No sequence has rows: nothing is written, by any of the calls but the lengths."""
    B = _B()
    case = Case([3000, 0], [rows, rows], 2, hd, 16, dtype, 51)
    pools = [p.to(DEV) for p in case.new_pools()]
    case.starts = [0, 0, 0]
    batch = case.batch(B, pools)
    q, k = (torch.ones(case.rows, h, hd, dtype=dtype, device=DEV) for h in (8, 2))
    before = [p.cpu().clone() for p in pools]
    out = torch.full_like(q, 77.0)
    B.ht_paged_attention(batch, q, *pools, case.anc().to(DEV), out=out)
    B.ht_paged_append(batch, q, k, k, *pools, q_out=out)
    ints = torch.zeros(case.rows, dtype=torch.int32, device=DEV)
    n, path, emitted, root, length = B.ht_paged_accept(batch, *pools, ints, ints, ints, 4)
    assert (out == 77.0).all() and n.tolist() == [0, 0] and root.tolist() == [-1, -1] and length.tolist() == [3000, 0]
    assert (path == -1).all() and (emitted == -1).all()
    as_int = torch.int16 if dtype == BF16 else torch.int32
    for p, x in zip(pools, before):
        assert torch.equal(p.cpu().view(as_int), x.view(as_int))


@pytest.mark.parametrize("dtype,rows", [(F32, 20), (BF16, 4), (BF16, 12), (BF16, 100)])
def test_two_calls_at_once(dtype, rows):
    """On two streams, each with scratch of its own: the bits of calls by themselves."""
    B = _B()
    cases = [Case([2500, 700], [rows, rows], 2, 128, 32, dtype, 52 + i) for i in range(2)]
    work = []
    for case in cases:
        pools = [p.to(DEV) for p in case.new_pools()]
        q = case.normal(case.rows, 8, 128).to(DEV)
        batch, anc = case.batch(B, pools), case.anc().to(DEV)
        work.append((batch, q, pools, anc, B.ht_paged_attention(batch, q, *pools, anc), B.ht_paged_attention_scratch(batch, 8), torch.cuda.Stream()))
        check(case, work[-1][4], q, pools, "alone")
    outs = [torch.empty_like(w[1]) for w in work]
    torch.cuda.synchronize()
    for _ in range(10):
        for o, (batch, q, pools, anc, _want, scratch, stream) in zip(outs, work):
            B.ht_paged_attention(batch, q, *pools, anc, out=o, scratch=scratch, stream=stream)
    torch.cuda.synchronize()
    for o, w in zip(outs, work):
        assert torch.equal(o, w[4])
