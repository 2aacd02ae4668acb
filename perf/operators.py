"""The operators of a batched decode step over a paged cache: what they are timed on, and their plain forms.

A batch of sequences keeps its keys and values in pages of a pool ([pages, kv heads, rows of a page, head dim], one pool for keys
and one for values); a table names the pages of every sequence in order.  A pass brings some rows for every sequence: one token, a
tree of drafted tokens, or a chunk of a prompt.

  append    norm of every query and key head (optional), rotary at the rows' positions, keys and values into their pages
  attention every row over its sequence's cached positions and over those rows of the pass that are it or its ancestors
  sample    one token per row of logits from given uniform numbers: temperature, top-k, top-p, min-p
  accept    the accepted path of every sequence's tree, and its rows moved to the front in the pages of every layer

Sizes are those of the repository's workloads (heads of 64 and 128; 4, 32 or 64 query heads; trees of 8 to 128 nodes; a vocabulary of
32000) and a larger vocabulary.
"""
import math

import torch

own = False

_EPS, _BASE = 1e-6, 10000.0
_MASK_WORDS = 4                      # 64-bit words of ancestor bits per row: up to 256 rows of a sequence in a pass


def listed():
    return [
        # one token each for a few short chats on a small model: the smallest call, latency
        dict(name="attention_small", kind="attention", seqs=4, rows=1, heads=4, kv_heads=4, head_dim=64, len=60, page=16,
             dtype="bf16", ragged=True, tree=False),
        # the fp32 model of the test configurations verifying its 8-node trees
        dict(name="attention_f32_trees", kind="attention", seqs=8, rows=8, heads=4, kv_heads=4, head_dim=64, len=190, page=16,
             dtype="f32", ragged=True, tree=True),
        # plain decoding of a full batch: one token for each of 32 requests of very different age
        dict(name="attention_tokens", kind="attention", seqs=32, rows=1, heads=32, kv_heads=32, head_dim=128, len=2048, page=16,
             dtype="bf16", ragged=True, tree=False),
        # one request with a very long history and shared key/value heads: few rows, a long axis
        dict(name="attention_long", kind="attention", seqs=1, rows=1, heads=64, kv_heads=8, head_dim=128, len=100003, page=64,
             dtype="bf16", ragged=False, tree=False),
        # the verify step of a batch: 64-node trees over long caches, eight query heads to a key head
        dict(name="attention_trees", kind="attention", seqs=8, rows=64, heads=64, kv_heads=8, head_dim=128, len=4096, page=64,
             dtype="bf16", ragged=True, tree=True),
        # one token each for many requests: norm of the heads, scaled positions over the whole head
        dict(name="append_tokens", kind="append", seqs=96, rows=1, heads=64, kv_heads=8, head_dim=128, len=700, page=16, dtype="bf16",
             ragged=True, tree=False, norm=True, rot=128, interleaved=False, scaled=True),
        # trees of a batch, interleaved pairs, half of the head rotated
        dict(name="append_trees", kind="append", seqs=16, rows=64, heads=32, kv_heads=32, head_dim=128, len=500, page=32, dtype="bf16",
             ragged=True, tree=True, norm=False, rot=64, interleaved=True, scaled=False),
        # the next token of one request
        dict(name="sample_one", kind="sample", rows=1, vocab=32000, dtype="f32", filters="all"),
        # a token after every node of a 64-node tree, nothing filtered: the whole distribution counts
        dict(name="sample_tree_unfiltered", kind="sample", rows=64, vocab=32000, dtype="f32", filters="none"),
        # a full batch over a large vocabulary, every row with settings of its own
        dict(name="sample_batch", kind="sample", rows=256, vocab=128001, dtype="bf16", filters="all"),
        # acceptance of a few small trees
        dict(name="accept_small", kind="accept", seqs=4, rows=8, layers=2, kv_heads=4, head_dim=64, len=100, page=16, dtype="f32",
             ragged=True),
        # acceptance of 64-node trees in every layer of a deep model
        dict(name="accept_trees", kind="accept", seqs=8, rows=64, layers=80, kv_heads=8, head_dim=128, len=120, page=64, dtype="bf16",
             ragged=True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "append", "sample", "accept"])
    heads, kv = rng.choice([(4, 4), (8, 2), (32, 32), (40, 40), (64, 8)])
    page = rng.choice([16, 32, 64, 128])
    if kind == "attention":
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        tree = rng.random() < 0.5
        rows = _log(rng, 2, 128) if tree else rng.choice([1, 1, _log(rng, 2, 64)])
        seqs = _log(rng, 1, 32)
        most = 2 ** 27 if dtype == "bf16" else 2 ** 23          # row, head, key triples: below the largest listed case
        length = _log(rng, 16, max(32, min(60000, most // (seqs * rows * heads), 2 ** 25 // (seqs * kv * 128))))
        return dict(kind=kind, seqs=seqs, rows=rows, heads=heads, kv_heads=kv, head_dim=64 if heads <= 8 else 128, len=length,
                    page=page, dtype=dtype, ragged=rng.random() < 0.7, tree=tree)
    if kind == "append":
        hd = rng.choice([64, 128])
        tree = rng.random() < 0.5
        return dict(kind=kind, seqs=_log(rng, 1, 64), rows=_log(rng, 2, 48) if tree else 1, heads=heads, kv_heads=min(kv, 8),
                    head_dim=hd, len=_log(rng, 10, 900), page=page, dtype=rng.choice(["f32", "bf16"]), ragged=rng.random() < 0.7,
                    tree=tree, norm=rng.random() < 0.5, rot=rng.choice([hd, hd // 2, hd // 4 + 2]), interleaved=rng.random() < 0.5,
                    scaled=rng.random() < 0.5)
    if kind == "sample":
        vocab = rng.choice([32000, _log(rng, 1000, 128001), _log(rng, 1000, 128001)])
        return dict(kind=kind, rows=_log(rng, 1, min(256, 2 ** 24 // vocab)), vocab=vocab, dtype=rng.choice(["f32", "bf16"]),
                    filters=rng.choice(["all", "all", "top_k", "top_p", "min_p", "none"]))
    return dict(kind=kind, seqs=_log(rng, 1, 8), rows=_log(rng, 2, 128), layers=_log(rng, 2, 48), kv_heads=min(kv, 8),
                head_dim=rng.choice([64, 128]), len=_log(rng, 10, 150), page=page, dtype=rng.choice(["f32", "bf16"]),
                ragged=rng.random() < 0.7)


# ------------------------------------------------------------------------------------------------ inputs
def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _lengths(c):
    """Cached positions of every sequence: ages spread evenly between one position and the longest."""
    if not c["ragged"]:
        return [c["len"]] * c["seqs"]
    return [c["len"] if b == 0 else 1 + int((c["len"] - 1) * (0.618034 * b % 1.0)) for b in range(c["seqs"])]


def _counts(c):
    """Rows of every sequence in this pass."""
    if not c["ragged"]:
        return [c["rows"]] * c["seqs"]
    return [c["rows"] if b == 0 else 1 + int((c["rows"] - 1) * (1.0 - 0.4 * (0.381966 * b % 1.0))) for b in range(c["seqs"])]


def _normal(g, shape, dtype, sigma=1.0, mean=0.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(sigma).add_(mean).to(dtype)


def _pages(c, g):
    """Row starts, lengths and a table of scattered pages; entries past a sequence's last page are -1."""
    lens, counts = _lengths(c), _counts(c)
    need = torch.tensor([-(-(n + t) // c["page"]) for n, t in zip(lens, counts)])
    width = -(-(c["len"] + c["rows"]) // c["page"])
    pool = int(need.sum()) + 3                                      # a few pages belong to nobody
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)[:int(need.sum())]
    table = torch.full((c["seqs"], width), -1, dtype=torch.int32, device="cuda")
    table[(torch.arange(width)[None, :] < need[:, None]).cuda()] = order
    starts = torch.tensor([0] + counts).cumsum(0).to(torch.int32).cuda()
    return dict(row_start=starts, length=torch.tensor(lens, dtype=torch.int32, device="cuda"), table=table, pool=pool,
                rows=sum(counts), max_rows=c["rows"], max_len=c["len"], page=c["page"])


def _trees(c, counts, cpu):
    """Parents of every sequence's rows, their depths and ancestor bits (on the host, as a scheduler keeps them)."""
    parents = [[-1] + [max(0, v - 1 - int(w * min(v, 6))) for v, w in zip(range(1, t), torch.rand(max(t - 1, 0), generator=cpu).tolist())]
               for t in counts]
    return [p for tree in parents for p in tree], parents


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    cpu = torch.Generator().manual_seed(seed + 1)
    if c["kind"] == "sample":
        rows, vocab = c["rows"], c["vocab"]
        z = _normal(g, (rows, vocab), torch.float32, 2.0)
        # what a trained head leaves: a few likely tokens far above the bulk, and on some rows tokens that a grammar rules out
        likely = torch.rand((rows, vocab), generator=g, device="cuda") < 40.0 / vocab
        z += likely * torch.rand((rows, vocab), generator=g, device="cuda") * 9.0
        ruled = torch.rand((rows, vocab), generator=g, device="cuda") < 0.3
        z.masked_fill_(ruled & (torch.arange(rows, device="cuda") % 5 == 4)[:, None], -math.inf)
        f = c["filters"]

        def settings(use, values, dtype):
            pick = torch.tensor(values, dtype=dtype)[torch.randint(len(values), (rows,), generator=cpu)]
            return pick.cuda() if f in ("all", use) else None

        return dict(case=c, logits=z.to(_type(c)), u=torch.rand(rows, generator=g, device="cuda"),
                    temperature=settings(f, [1.0, 0.7, 0.9, 1.2, 0.0] if f == "all" else [1.0, 0.8], torch.float32),
                    top_k=settings("top_k", [0, 40, 50, 200, 1000] if f == "all" else [40, 1000], torch.int32),
                    top_p=settings("top_p", [1.0, 0.9, 0.95, 0.8], torch.float32),
                    min_p=settings("min_p", [0.0, 0.05, 0.02], torch.float32))
    counts = _counts(c)
    s = dict(case=c, **_pages(c, g))
    kv, hd, t = c["kv_heads"], c["head_dim"], _type(c)
    shape = (s["pool"], kv, c["page"], hd)
    if c["kind"] == "accept":
        shape = (c["layers"],) + shape
    s["k_pages"], s["v_pages"] = _normal(g, shape, t), _normal(g, shape, t)
    if c.get("tree", c["kind"] == "accept"):
        flat, parents = _trees(c, counts, cpu)
        depth, bits = [], []
        for tree in parents:
            d, up = [], []
            for v, p in enumerate(tree):
                d.append(0 if p < 0 else d[p] + 1)
                up.append((0 if p < 0 else up[p]) | 1 << v)
            depth += d
            bits += [[w - (1 << 64) if w >> 63 else w for w in (u >> 64 * i & (1 << 64) - 1 for i in range(_MASK_WORDS))] for u in up]
        s["parent"] = torch.tensor(flat, dtype=torch.int32, device="cuda")
        s["depth"] = torch.tensor(depth, dtype=torch.int32, device="cuda")
        s["anc"] = torch.tensor(bits, dtype=torch.int64, device="cuda")
    else:
        s["parent"] = s["depth"] = s["anc"] = None
    if c["kind"] == "attention":
        s["q"] = _normal(g, (s["rows"], c["heads"], hd), t, 1.5)
    elif c["kind"] == "append":
        # the projections of a block leave q, k and v of a row side by side
        qkv = _normal(g, (s["rows"], c["heads"] + 2 * kv, hd), t)
        s["q"], s["k"], s["v"] = qkv[:, :c["heads"]], qkv[:, c["heads"]:c["heads"] + kv], qkv[:, c["heads"] + kv:]
        s["q_gain"] = _normal(g, (hd,), t, 0.1, 1.0) if c["norm"] else None
        s["k_gain"] = _normal(g, (hd,), t, 0.1, 1.0) if c["norm"] else None
        s["inv_freq"], s["amplitude"] = None, 1.0
        if c["scaled"]:
            # frequencies of a context stretched eightfold: the slow ones divided by eight, the fast ones kept, a ramp between
            j = torch.arange(c["rot"] // 2, dtype=torch.float64)
            f = _BASE ** (-2.0 * j / c["rot"])
            keep = ((f * 4096 / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
            s["inv_freq"], s["amplitude"] = (f * keep + f / 8 * (1 - keep)).float().cuda(), 0.1 * math.log(8.0) + 1.0
    else:
        # tokens of the trees, and what the model answered after every node: mostly one of the drafted children
        tok, ans, at = [], [], 0
        for tree in parents:
            own_tok = torch.randint(32000, (len(tree),), generator=cpu).tolist()
            answer = torch.randint(32000, (len(tree),), generator=cpu).tolist()
            for v in range(len(tree)):
                kids = [u for u in range(v + 1, len(tree)) if tree[u] == v]
                if kids and float(torch.rand((), generator=cpu)) < 0.8:
                    answer[v] = own_tok[kids[int(torch.randint(len(kids), (), generator=cpu))]]
            tok += own_tok
            ans += answer
        s["tokens"] = torch.tensor(tok, dtype=torch.int32, device="cuda")
        s["answers"] = torch.tensor(ans, dtype=torch.int32, device="cuda")
        s["max_path"] = min(16, c["rows"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _place(s):
    """Sequence and place in it of every row."""
    starts = s["row_start"].long()
    row = torch.arange(s["rows"], device="cuda")
    seq = torch.searchsorted(starts, row, right=True) - 1
    return seq, row - starts[seq]


def _seen(s, J):
    """[rows, J]: whether a row sees the position of its sequence."""
    seq, at = _place(s)
    n = s["length"].long()[seq][:, None]
    j = torch.arange(J, device="cuda")[None, :]
    u = (j - n).clamp(0, 64 * _MASK_WORDS - 1)
    if s["anc"] is None:
        mine = u <= at[:, None]
    else:
        mine = (s["anc"].gather(1, u >> 6) >> (u & 63) & 1).bool()
    count = (s["row_start"][1:] - s["row_start"][:-1]).long()[seq][:, None]
    return (j < n) | (j - n < count) & (j >= n) & mine


def _plain_attention(s):
    c = s["case"]
    B, R, kv, hd = c["seqs"], s["max_rows"], c["kv_heads"], c["head_dim"]
    G, J = c["heads"] // kv, s["max_len"] + R
    slot = torch.arange(J, device="cuda")
    page = s["table"].long()[:, slot // s["page"]].clamp(min=0)                     # [B, J]
    k = s["k_pages"][page, :, (slot % s["page"])[None, :]].float().transpose(1, 2).contiguous()      # [B, kv, J, hd]
    v = s["v_pages"][page, :, (slot % s["page"])[None, :]].float().transpose(1, 2).contiguous()
    seq, at = _place(s)
    q = torch.zeros(B, R, c["heads"], hd, device="cuda")
    q[seq, at] = s["q"].float()
    q = q.view(B, R, kv, G, hd).transpose(1, 2).reshape(B, kv, R * G, hd)
    seen = torch.zeros(B, R, J, dtype=torch.bool, device="cuda")
    seen[seq, at] = _seen(s, J)
    seen = seen[:, None, :, None, :].expand(B, 1, R, G, J).reshape(B, 1, R * G, J)
    z = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(hd)).masked_fill_(~seen, -math.inf)
    top = z.amax(3, keepdim=True)
    e = z.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = e.sum(3, keepdim=True)
    o = torch.matmul(e, v) / torch.where(total == 0, 1.0, total)
    o = o.view(B, kv, R, G, hd).transpose(1, 2).reshape(B, R, c["heads"], hd)
    return o[seq, at].to(_type(c))


def _angles(s, pos):
    c = s["case"]
    f = s["inv_freq"].double() if s["inv_freq"] is not None else \
        _BASE ** (-2.0 * torch.arange(c["rot"] // 2, dtype=torch.float64, device="cuda") / c["rot"])
    t = pos.double()[:, None] * f
    return (torch.cos(t) * s["amplitude"]).float()[:, None, :], (torch.sin(t) * s["amplitude"]).float()[:, None, :]


def _plain_turn(s, x, gain, co, si):
    c = s["case"]
    x = x.float()
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(2, keepdim=True) + _EPS) * gain.float()
    r = c["rot"]
    head, rest = x[..., :r], x[..., r:]
    if c["interleaved"]:
        a, b = head[..., 0::2], head[..., 1::2]
        head = torch.stack([a * co - b * si, b * co + a * si], dim=3).flatten(2)
    else:
        a, b = head[..., :r // 2], head[..., r // 2:]
        head = torch.cat([a * co - b * si, b * co + a * si], dim=2)
    return torch.cat([head, rest], dim=2).to(_type(c))


def _plain_append(s):
    seq, at = _place(s)
    n = s["length"].long()[seq]
    co, si = _angles(s, n + (at if s["depth"] is None else s["depth"].long()))
    q = _plain_turn(s, s["q"], s["q_gain"], co, si)
    slot = n + at
    page = s["table"].long()[seq, slot // s["page"]]
    s["k_pages"][page, :, slot % s["page"]] = _plain_turn(s, s["k"], s["k_gain"], co, si)
    s["v_pages"][page, :, slot % s["page"]] = s["v"]
    return dict(q=q, k_pages=s["k_pages"], v_pages=s["v_pages"])


def _plain_sample(s):
    # 64 bits throughout: which token a number falls on is decided next to borders
    x = s["logits"].double()
    x = torch.where(x.isnan(), -math.inf, x)
    rows, vocab = x.shape
    top = x.amax(1, keepdim=True)
    T = torch.ones(rows, 1, dtype=torch.float64, device="cuda") if s["temperature"] is None else s["temperature"].double()[:, None]
    greedy = ~(T > 0)
    e = torch.where(x == -math.inf, 0.0, torch.where(x == top, 1.0, ((x - top) / torch.where(greedy, 1.0, T)).exp()))
    keep = torch.ones_like(x, dtype=torch.bool)
    if s["top_k"] is not None or s["top_p"] is not None:
        order = torch.sort(x, dim=1, descending=True, stable=True).indices          # ties: lowest index first
        e_sorted = e.gather(1, order)
        rank = torch.arange(vocab, device="cuda")[None, :]
        kept = torch.ones_like(keep)
        if s["top_k"] is not None:
            k = s["top_k"].long()[:, None]
            kept = (rank < k) | (k <= 0)
        if s["top_p"] is not None:
            p = s["top_p"].double()[:, None]
            mass = (e_sorted * kept).cumsum(1)
            before = mass - e_sorted * kept
            kept = kept & ((before < p * mass[:, -1:]) | (p >= 1) | (rank == 0))
        keep = torch.zeros_like(keep).scatter_(1, order, kept)
    if s["min_p"] is not None:
        keep = keep & (e >= s["min_p"].double()[:, None])
    e = e * keep
    cum = e.cumsum(1)
    total = cum[:, -1:]
    past = (cum <= s["u"].double()[:, None] * total).sum(1)
    last = torch.where(e > 0, torch.arange(vocab, device="cuda")[None, :], 0).amax(1)
    token = torch.minimum(past, last)
    logprob = (e.gather(1, token[:, None]) / total).log()[:, 0]
    first = torch.where(x == top, torch.arange(vocab, device="cuda")[None, :], vocab).amin(1)
    token, logprob = torch.where(greedy[:, 0], first, token), torch.where(greedy[:, 0], 0.0, logprob)
    return dict(tokens=token.to(torch.int32), logprob=logprob.float())


def _plain_accept(s):
    c = s["case"]
    B, R, P = c["seqs"], s["max_rows"], s["max_path"]
    seq, at = _place(s)
    up = torch.full((B, R), -2, dtype=torch.long, device="cuda")
    tok, ans, bits = torch.zeros_like(up), torch.zeros_like(up), torch.zeros(B, R, _MASK_WORDS, dtype=torch.long, device="cuda")
    up[seq, at], tok[seq, at], ans[seq, at], bits[seq, at] = s["parent"].long(), s["tokens"].long(), s["answers"].long(), s["anc"]
    node = torch.arange(R, device="cuda")
    # a node is answered if its parent's answer is its token and no sibling before it has the same
    right = (up >= 0) & (ans.gather(1, up.clamp(min=0)) == tok)
    earlier = ((up[:, :, None] == up[:, None, :]) & right[:, None, :] & (node[None, :] < node[:, None])).any(2)
    right = right & ~earlier | (up == -1)
    line = (bits[:, :, node >> 6] >> (node & 63) & 1).bool()                        # [B, node, ancestor-or-self]
    taken = (up >= -1) & ~(line & ~right[:, None, :]).any(2)
    step = taken.long().cumsum(1) - 1
    taken &= step < P
    count = taken.sum(1)
    path = torch.full((B, P), -1, dtype=torch.long, device="cuda")
    b, v = taken.nonzero(as_tuple=True)
    path[b, step[b, v]] = v
    n = s["length"].long()
    src, dst = n[b] + v, n[b] + step[b, v]
    table = s["table"].long()
    for pool in (s["k_pages"], s["v_pages"]):
        rows = pool[:, table[b, src // s["page"]], :, src % s["page"]]
        pool[:, table[b, dst // s["page"]], :, dst % s["page"]] = rows
    have = path >= 0
    emitted = torch.where(have, tok.gather(1, path.clamp(min=0)), -1)
    last = path.gather(1, (count - 1)[:, None]).clamp(min=0)
    return dict(accepted=count.int(), path=path.int(), tokens=emitted.int(), next_root=ans.gather(1, last)[:, 0].int(),
                length=(n + count).int(), k_pages=s["k_pages"], v_pages=s["v_pages"])


# ------------------------------------------------------------------------------------------------ one pass
def _own(s):
    import paper_2404_12022_amd.binding as B
    c = s["case"]
    if c["kind"] == "sample":
        tokens, logprob = B.ht_sample_rows(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
        return dict(tokens=tokens, logprob=logprob)
    batch = s.get("batch")
    if batch is None:                                    # the description of the batch's buffers, kept as long as they are
        batch = s["batch"] = B.PagedBatch(s["row_start"], s["length"], s["table"], s["k_pages"], s["v_pages"], s["rows"],
                                          s["max_rows"], s["max_len"])
    if c["kind"] == "attention":
        if "scratch" not in s:
            s["scratch"] = B.ht_paged_attention_scratch(batch, c["heads"])
        return B.ht_paged_attention(batch, s["q"], s["k_pages"], s["v_pages"], s["anc"], scratch=s["scratch"])
    if c["kind"] == "append":
        q = B.ht_paged_append(batch, s["q"], s["k"], s["v"], s["k_pages"], s["v_pages"], depth=s["depth"], q_gain=s["q_gain"],
                              k_gain=s["k_gain"], eps=_EPS, rot=c["rot"], interleaved=c["interleaved"], rope_base=_BASE,
                              inv_freq=s["inv_freq"], amplitude=s["amplitude"])
        return dict(q=q, k_pages=s["k_pages"], v_pages=s["v_pages"])
    accepted, path, tokens, root, length = B.ht_paged_accept(batch, s["k_pages"], s["v_pages"], s["parent"], s["tokens"], s["answers"],
                                                             s["max_path"])
    return dict(accepted=accepted, path=path, tokens=tokens, next_root=root, length=length, k_pages=s["k_pages"], v_pages=s["v_pages"])


def run(state):
    if own:
        return _own(state)
    return {"attention": _plain_attention, "append": _plain_append, "sample": _plain_sample, "accept": _plain_accept}[state["case"]["kind"]](state)


def work(case):
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "sample":
        return {"bytes": c["rows"] * (c["vocab"] * size + 28), "flops": 3 * c["rows"] * c["vocab"]}
    lens, counts = _lengths(c), _counts(c)
    kv, hd = c["kv_heads"], c["head_dim"]
    rows = sum(counts)
    if c["kind"] == "attention":
        keys = sum(n + t for n, t in zip(lens, counts))
        pairs = sum(t * n + (t * 5 if c["tree"] else t * (t + 1) // 2) for n, t in zip(lens, counts))
        return {"bytes": size * hd * (2 * kv * keys + 2 * rows * c["heads"]), "flops": 4 * hd * c["heads"] * pairs}
    if c["kind"] == "append":
        return {"bytes": 2 * size * rows * hd * (c["heads"] + 2 * kv), "flops": 8 * rows * hd * (c["heads"] + kv)}
    return {"bytes": 4 * size * kv * hd * c["layers"] * c["seqs"] * 3 + 12 * rows, "flops": 8 * rows}       # three rows move, or so


# ------------------------------------------------------------------------------------------------ 64 bits, from the definitions
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "sample":
        return _exact_sample(s)
    lens, counts = _lengths(c), _counts(c)
    table, P, hd, kv = s["table"].cpu(), c["page"], c["head_dim"], c["kv_heads"]
    at = 0
    if c["kind"] == "attention":
        G, out, parent = c["heads"] // kv, [], None if s["parent"] is None else s["parent"].tolist()
        for b, (n, t) in enumerate(zip(lens, counts)):
            used = table[b, :-(-(n + t) // P)].long().cuda()
            k = s["k_pages"][used].transpose(1, 2).reshape(-1, kv, hd)[:n + t].double()
            v = s["v_pages"][used].transpose(1, 2).reshape(-1, kv, hd)[:n + t].double()
            seen = torch.ones(t, n + t, dtype=torch.bool)
            for r in range(t):
                line, v0 = set(range(r + 1)), r
                if parent is not None:
                    line = set()
                    while v0 >= 0:
                        line.add(v0)
                        v0 = parent[at + v0]
                seen[r, n:] = torch.tensor([u in line for u in range(t)])
            seen, o = seen.cuda(), torch.empty(t, c["heads"], hd, dtype=torch.float64, device="cuda")
            for h in range(c["heads"]):
                z = (s["q"][at:at + t, h].double() @ k[:, h // G].T.contiguous()) / math.sqrt(hd)
                z = z.masked_fill(~seen, -math.inf)
                w = (z - z.amax(1, keepdim=True)).exp()
                o[:, h] = (w @ v[:, h // G].contiguous()) / w.sum(1, keepdim=True)
            out.append(o)
            at += t
        return torch.cat(out)
    if c["kind"] == "append":
        k_pages, v_pages, q = s["k_pages"].double(), s["v_pages"].double(), []
        f = s["inv_freq"].double().cpu() if c["scaled"] else \
            torch.tensor([_BASE ** (-2.0 * j / c["rot"]) for j in range(c["rot"] // 2)], dtype=torch.float64)
        depth = None if s["depth"] is None else s["depth"].cpu()
        gains = [None if x is None else x.double().cpu() for x in (s["q_gain"], s["k_gain"])]
        rows_q, rows_k, rows_v = (s[x].double().cpu() for x in "qkv")
        low = torch.arange(c["rot"] // 2) * (2 if c["interleaved"] else 1)
        high = low + (1 if c["interleaved"] else c["rot"] // 2)

        def turn(x, gain, pos):
            if gain is not None:
                x = x / (x.square().mean(1, keepdim=True) + _EPS).sqrt() * gain
            y, a, b = x.clone(), x[:, low], x[:, high]
            y[:, low] = s["amplitude"] * (a * torch.cos(pos * f) - b * torch.sin(pos * f))
            y[:, high] = s["amplitude"] * (b * torch.cos(pos * f) + a * torch.sin(pos * f))
            return y

        for b, (n, t) in enumerate(zip(lens, counts)):
            for i in range(t):
                pos = n + (i if depth is None else int(depth[at]))
                page, row = int(table[b, (n + i) // P]), (n + i) % P
                q.append(turn(rows_q[at], gains[0], pos))
                k_pages[page, :, row] = turn(rows_k[at], gains[1], pos).cuda()
                v_pages[page, :, row] = rows_v[at].cuda()
                at += 1
        return dict(q=torch.stack(q), k_pages=k_pages, v_pages=v_pages)
    parent, tok, ans = (s[x].tolist() for x in ("parent", "tokens", "answers"))
    k_pages, v_pages = s["k_pages"], s["v_pages"]
    found = dict(accepted=[], path=[], tokens=[], next_root=[], length=[])
    for b, (n, t) in enumerate(zip(lens, counts)):
        path = [0]
        while len(path) < s["max_path"]:
            kids = [u for u in range(t) if parent[at + u] == path[-1] and tok[at + u] == ans[at + path[-1]]]
            if not kids:
                break
            path.append(kids[0])
        for j, v in enumerate(path):
            a, z = n + v, n + j
            for pool in (k_pages, v_pages):
                pool[:, int(table[b, z // P]), :, z % P] = pool[:, int(table[b, a // P]), :, a % P]
        rest = [-1] * (s["max_path"] - len(path))
        found["accepted"].append(len(path))
        found["path"].append(path + rest)
        found["tokens"].append([tok[at + v] for v in path] + rest)
        found["next_root"].append(ans[at + path[-1]])
        found["length"].append(n + len(path))
        at += t
    return dict({x: torch.tensor(y, dtype=torch.int32) for x, y in found.items()}, k_pages=k_pages, v_pages=v_pages)


def _exact_sample(s):
    z, u = s["logits"].double().cpu().numpy(), s["u"].double().cpu().numpy()
    T, K, P, M = (None if s[x] is None else s[x].double().cpu().numpy() for x in ("temperature", "top_k", "top_p", "min_p"))
    import numpy as np
    tokens, logprob = [], []
    for r in range(z.shape[0]):
        x, t = z[r], 1.0 if T is None else T[r]
        if t <= 0:
            tokens.append(int(np.argmax(x)))
            logprob.append(0.0)
            continue
        e = np.exp((x - x.max()) / t)
        left = np.argsort(-x, kind="stable")
        if K is not None and K[r] > 0:
            left = left[:int(K[r])]
        if P is not None and P[r] < 1:
            mass = np.cumsum(e[left])
            left = left[:int(np.searchsorted(mass, P[r] * mass[-1], side="left")) + 1]
        if M is not None:
            left = left[e[left] >= M[r]]
        left = np.sort(left)
        mass = np.cumsum(e[left])
        at = min(int(np.searchsorted(mass, u[r] * mass[-1], side="right")), len(left) - 1)
        tokens.append(int(left[at]))
        logprob.append(float(np.log(e[left[at]] / mass[-1])))
    return dict(tokens=torch.tensor(tokens, dtype=torch.int32), logprob=torch.tensor(logprob, dtype=torch.float64))
