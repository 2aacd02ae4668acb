"""CPU-only: what the entry points over pages and the sampler refuse, before anything reaches a GPU."""
import ctypes as C
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if not os.path.exists(os.path.join(ROOT, "paper_2404_12022_amd", "libht.so")):
    pytest.skip("library not built", allow_module_level=True)

import paper_2404_12022_amd.binding as B

P = 1 << 20            # an address that nothing follows: every call here fails before it would
FAR = 1 << 30


def batch(**kw):
    b = B.ht_paged_batch(4, 40, 16, 100, 2, 64, B.HT_BF16, 16, 50, 8, P, P, P)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def turn(**kw):
    t = B.ht_head_turn(None, None, 1e-6, 64, 0, 10000.0, None, 1.0)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def code(name, *args):
    rc = getattr(B.lib, name)(*args)
    assert rc == B.HT_OK or B.lib.ht_last_error()
    return rc


BAD = [dict(seqs=0), dict(seqs=65536), dict(rows=0), dict(max_rows=0), dict(max_rows=257), dict(max_len=-1), dict(max_len=(1 << 30) + 1),
       dict(n_kv_heads=0), dict(head_dim=0), dict(head_dim=63), dict(head_dim=258), dict(dtype=2), dict(page_rows=0), dict(page_rows=4),
       dict(page_rows=24), dict(page_rows=8192), dict(n_pages=0), dict(table_width=0), dict(row_start=None), dict(len=None),
       dict(page_table=None)]


@pytest.mark.parametrize("bad", BAD, ids=lambda d: "%s=%s" % next(iter(d.items())))
def test_a_bad_batch_is_refused_everywhere(bad):
    b = C.byref(batch(**bad))
    assert code("ht_tree_tables", b, P, P, P, None) == B.HT_EINVAL
    assert code("ht_paged_append", b, C.byref(turn()), 4, P, FAR, P, FAR, P, FAR, None, P, FAR, P, P, None) == B.HT_EINVAL
    assert code("ht_paged_attention", b, 4, P, FAR, P, P, None, 0.0, P, FAR, P, FAR, None) == B.HT_EINVAL
    assert B.lib.ht_paged_attention_scratch_bytes(b, 4) == 0
    assert code("ht_paged_accept", b, 1, 0, P, P, P, P, P, 4, FAR, FAR, FAR, FAR, FAR, None) == B.HT_EINVAL


def test_a_table_that_is_too_short_is_refused():
    b = C.byref(batch(max_len=8 * 16 - 16 + 1))
    assert code("ht_tree_tables", b, P, P, P, None) == B.HT_ECAPACITY
    assert code("ht_paged_append", b, C.byref(turn()), 4, P, FAR, P, FAR, P, FAR, None, P, FAR, P, P, None) == B.HT_ECAPACITY
    assert code("ht_paged_attention", b, 4, P, FAR, P, P, None, 0.0, P, FAR, P, FAR, None) == B.HT_ECAPACITY
    assert B.lib.ht_paged_attention_scratch_bytes(b, 4) == 0
    assert code("ht_paged_accept", b, 1, 0, P, P, P, P, P, 4, FAR, FAR, FAR, FAR, FAR, None) == B.HT_ECAPACITY
    assert B.lib.ht_paged_attention_scratch_bytes(C.byref(batch(max_len=8 * 16 - 16)), 4) > 0


def test_append_refuses():
    ok = dict(t=turn(), Hq=4, q=P, qs=256, k=P, ks=128, v=P, vs=128, depth=None, out=P, os=256, kp=P, vp=P)

    def call(**kw):
        a = dict(ok, **kw)
        t = None if a["t"] is None else C.byref(a["t"])
        return code("ht_paged_append", C.byref(batch()), t, *[a[n] for n in ("Hq", "q", "qs", "k", "ks", "v", "vs", "depth", "out", "os", "kp", "vp")], None)

    for bad in (dict(t=None), dict(Hq=0), dict(Hq=3), dict(q=None, k=None, v=None), dict(v=None), dict(k=None), dict(out=None), dict(kp=None), dict(vp=None),
                dict(qs=255), dict(os=255), dict(ks=127), dict(vs=127), dict(t=turn(rot_dim=-2)), dict(t=turn(rot_dim=3)),
                dict(t=turn(rot_dim=66)), dict(t=turn(rope_base=1.0)), dict(t=turn(rope_base=float("nan"))), dict(t=turn(q_gain=P, eps=-1.0))):
        assert call(**bad) == B.HT_EINVAL, bad


def test_attention_refuses():
    b = batch()
    need = B.lib.ht_paged_attention_scratch_bytes(C.byref(b), 4)
    assert need > 0
    ok = dict(Hq=4, q=P, qs=256, kp=P, vp=P, anc=None, scale=0.0, out=P, os=256, s=P, sb=need)

    def call(**kw):
        a = dict(ok, **kw)
        return code("ht_paged_attention", C.byref(b), *[a[n] for n in ("Hq", "q", "qs", "kp", "vp", "anc", "scale", "out", "os", "s", "sb")], None)

    for bad in (dict(Hq=0), dict(Hq=5), dict(q=None), dict(kp=None), dict(vp=None), dict(out=None), dict(s=None), dict(qs=255), dict(os=255),
                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(sb=need - 1), dict(s=P + 64)):
        assert call(**bad) == B.HT_EINVAL, bad


def test_pages_of_attention_lie_on_16_bytes_and_groups_end_at_256():
    b = batch(n_kv_heads=1)
    need = B.lib.ht_paged_attention_scratch_bytes(C.byref(b), 256)
    assert need > 0 and B.lib.ht_paged_attention_scratch_bytes(C.byref(b), 257) == 0
    call = lambda Hq, kp, vp: code("ht_paged_attention", C.byref(b), Hq, P, FAR, kp, vp, None, 0.0, P, FAR, P, FAR, None)  # noqa: E731
    assert call(257, P, P) == call(4, P + 8, P) == call(4, P, P + 2) == B.HT_EINVAL
    assert code("ht_paged_append", C.byref(b), C.byref(turn()), 257, P, FAR, P, FAR, P, FAR, None, P, FAR, P, P, None) == B.HT_EINVAL


def test_sampling_refuses():
    ok = dict(z=P, stride=100, dtype=B.HT_F32, rows=3, V=100, u=P, tok=P)

    def call(**kw):
        a = dict(ok, **kw)
        return code("ht_sample_rows", a["z"], a["stride"], a["dtype"], a["rows"], a["V"], a["u"], None, None, None, None, a["tok"], None, None)

    for bad in (dict(z=None), dict(u=None), dict(tok=None), dict(dtype=7), dict(rows=0), dict(rows=(1 << 20) + 1), dict(V=0), dict(stride=99),
                dict(V=B.HT_MAX_SAMPLE_VOCAB + 1, stride=FAR)):
        assert call(**bad) == B.HT_EINVAL, bad


def test_acceptance_refuses():
    ok = dict(layers=2, ls=50 * 2 * 16 * 64, kp=P, vp=P, par=P, tok=P, ans=P, mp=4, n=FAR, path=FAR, em=FAR, root=FAR, new=FAR)

    def call(**kw):
        a = dict(ok, **kw)
        return code("ht_paged_accept", C.byref(batch(len=3 * P, row_start=4 * P)),
                    *[a[n] for n in ("layers", "ls", "kp", "vp", "par", "tok", "ans", "mp", "n", "path", "em", "root", "new")], None)

    for bad in ([{n: None} for n in ("kp", "vp", "par", "tok", "ans", "n", "path", "em", "root", "new")] +
                [dict(layers=0), dict(layers=65536), dict(ls=50 * 2 * 16 * 64 - 1), dict(mp=0), dict(mp=257), dict(new=3 * P), dict(new=3 * P + 12),
                 dict(root=P + 4 * 39), dict(path=3 * P - 4 * 15), dict(n=4 * P + 16), dict(em=P)]):
        assert call(**bad) == B.HT_EINVAL, bad


def test_the_binding_refuses_what_is_not_on_the_gpu():
    z = torch.zeros(3, 10)
    with pytest.raises(B.HTError) as e:
        B.ht_sample_rows(z, torch.zeros(3))
    assert e.value.code == B.HT_EINVAL
    pages = torch.zeros(4, 2, 16, 64)
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(B.HTError) as e:
        B.PagedBatch(i(3), i(2), i(2, 4), pages, pages, 5, 3, 20)
    assert e.value.code == B.HT_EINVAL


def test_the_limit_of_the_vocabulary_matches_the_header():
    text = open(os.path.join(ROOT, "include", "ht.h")).read()
    assert "HT_MAX_SAMPLE_VOCAB = 1 << 20" in text and B.HT_MAX_SAMPLE_VOCAB == 1 << 20
