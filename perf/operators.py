"""What the paged cache and the attention over it are measured on.

A case is one pass of an operator of the paged cache (pages of ``page`` tokens
that the rows of a page table share, every layer of a token under one page
number):

* ``fork``     rows are dropped, branched again from other rows and extended:
               page counts, tables, and the copy of each shared last page;
* ``compact``  a branch of each row keeps the tokens that a selection names and
               its recent window, in pages of its own;
* ``move``     new tokens go into the pages, and (``load``) back out of them;
* ``tree``     attention of drafted tokens over the cache, a drafted token
               seeing the others through a bit mask;
* ``sink``     attention with a sliding window and a few first tokens that stay
               visible, for one new token or a chunk of them.

The shapes are the repository's workloads (28 query and 4 KV heads, or 32 and
8; caches of 5 and 20 screenshots before and after their compression; batches
of ragged lengths) with pages of 16 to 128 tokens in shuffled order.  Keys,
values and queries are normal; the first four keys and all queries share a
direction, so that the first tokens take more of the mass, as they do in real
caches.  What is copied is compared as 16-bit words.
"""
import math
import random

import torch

own = False
D = 128     # head dimension
DEV = "cuda"


def _case(name, op, **over):
    c = dict(name=name, op=op, heads=28, kv_heads=4, layers=2, page=64, n=1, ctx=2736, ragged=False, T=1)
    c.update(over)
    return c


def listed():
    return [
        # four branches of one compressed trajectory, each about to append its own token
        _case("fork_beams", "fork", layers=28, n=4, sources=1, ctx=2737),
        # serving: 64 rows branched from 16 five-screenshot caches of many lengths
        _case("fork_64", "fork", layers=28, n=64, sources=16, ctx=14033, ragged=True, T=3),
        # one step's compression of a five-screenshot cache, 2704 tokens and the window kept
        _case("compact_5shot", "compact", layers=28, ctx=14032, budget=2704, window=32, per_head=False),
        # eight trajectories of many lengths, each KV head with tokens of its own
        _case("compact_ragged_8", "compact", layers=28, n=8, ctx=12001, ragged=True, page=16, budget=2048, window=32,
              per_head=True),
        # serving: one layer's new token of 64 rows
        _case("move_decode_64", "move", n=64, ctx=2801, ragged=True, page=16, load=False),
        # a compressed cache goes into pages, every layer, and comes back for the next scoring
        _case("move_prompt_28l", "move", layers=28, ctx=2736, T=2736, load=True),
        # one trajectory checks eight drafted tokens over its compressed cache
        _case("tree_first", "tree", ctx=2744, T=8),
        # serving: 32 rows of many lengths, 26 drafted tokens each
        _case("tree_32", "tree", n=32, ctx=14033, ragged=True, T=26),
        # four 20-screenshot caches, the widest tree
        _case("tree_long", "tree", n=4, ctx=56193, page=128, T=64),
        # the smallest call: one token of a short cache
        _case("sink_tiny", "sink", ctx=577, sinks=4, window=512),
        # serving: 64 rows of many lengths, one token each
        _case("sink_decode_64", "sink", heads=32, kv_heads=8, n=64, ctx=14033, ragged=True, page=32, sinks=4,
              window=4096),
        # one screenshot's tokens appended at once
        _case("sink_chunk", "sink", ctx=8113, T=2704, sinks=64, window=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["fork", "compact", "move", "tree", "tree", "sink", "sink"])
    heads, kv_heads = rng.choice([(28, 4), (28, 4), (32, 8), (16, 2), (8, 8), (40, 8), (12, 1)])
    c = _case("", op, heads=heads, kv_heads=kv_heads, page=rng.choice([16, 32, 64, 64, 128]),
              ctx=_log(rng, 600, 14000), ragged=rng.random() < 0.6)
    del c["name"]
    if op == "fork":
        c.update(layers=_log(rng, 1, 28), n=_log(rng, 1, 64), T=_log(rng, 1, 200))
        c["sources"] = rng.randint(1, min(16, c["n"]))
    elif op == "compact":
        c.update(layers=_log(rng, 1, 28), n=_log(rng, 1, 8), window=rng.choice([8, 16, 32]),
                 per_head=rng.random() < 0.3)
        while heads // kv_heads * c["window"] > 256:
            c["window"] //= 2
        c["budget"] = _log(rng, 50, max(51, c["ctx"] // 2))
    elif op == "move":
        c.update(layers=_log(rng, 1, 28), n=_log(rng, 1, 32), load=rng.random() < 0.5)
        c["T"] = _log(rng, 1, c["ctx"] // 4)
    elif op == "tree":
        c.update(n=_log(rng, 1, 32), T=rng.randint(1, 64))
    else:
        c.update(n=_log(rng, 1, 64), sinks=rng.choice([0, 1, 4, 64]), window=_log(rng, 64, 16384))
        c["T"] = rng.choice([1, 1, _log(rng, 2, 256)])
    while c["n"] > 1 and _cost(c) > _MOST[op]:
        c["n"] -= 1
        if op == "fork":
            c["sources"] = min(c["sources"], c["n"])
    while c["T"] > 1 and op not in ("tree",) and _cost(c) > _MOST[op]:
        c["T"] = c["T"] // 2
    return c


def _cost(c):
    w = work(dict(c, name=""))
    return max(w["bytes"], w["flops"] / 50)


_MOST = dict(fork=235e6, compact=1e9, move=300e6, tree=2e9, sink=2e9)


def _lens(c):
    """Tokens of each row before the call: they depend on the case alone.  A row is at least a quarter
    of the longest, and long enough for the call."""
    rng = random.Random(c["ctx"] * 131 + c["n"])
    least = {"compact": c.get("budget", 0) + c.get("window", 0), "fork": 1}.get(c["op"], c["T"])
    rows = c.get("sources", c["n"])
    return [max(least, rng.randint(c["ctx"] // 4, c["ctx"]) if c["ragged"] and i else c["ctx"]) for i in range(rows)]


def _queries(c):
    """Real queries (new tokens) of each row: all T, or fewer behind the first of a ragged batch."""
    rng = random.Random(c["T"] * 17 + c["n"])
    return [rng.randint(max(1, c["T"] // 2), c["T"]) if c["ragged"] and i else c["T"] for i in range(c["n"])]


def _ceil(a, b):
    return -(-a // b)


def work(c):
    row = c["kv_heads"] * D * 2      # bytes of one token's K (or V) in a layer
    lens = _lens(c)
    if c["op"] == "fork":
        b = 0.0
        for i in range(c["n"]):
            length = lens[i % c["sources"]]
            b += 4 * (length % c["page"]) * row * c["layers"]          # the shared last page, K and V, read and written
            b += 4 * 4 * _ceil(length + c["T"], c["page"]) + 24         # table and counts, read and written
        return {"bytes": b, "flops": 0}
    if c["op"] == "compact":
        sets = c["kv_heads"] if c["per_head"] else 1
        kept = c["budget"] + c["window"]
        b = c["n"] * c["layers"] * (4 * kept * row + 4 * sets * c["budget"] + 8 * sets * kept)
        b += sum(4 * 4 * (_ceil(n, c["page"]) + _ceil(kept, c["page"])) for n in lens)
        return {"bytes": b, "flops": 0}
    if c["op"] == "move":
        return {"bytes": sum(_queries(c)) * c["layers"] * row * (8 if c["load"] else 4) + 4 * sum(_ceil(t, c["page"]) for t in _queries(c)),
                "flops": 0}
    qs = _queries(c)
    io = sum(qs) * c["heads"] * (D * 4 + 4)
    if c["op"] == "tree":
        return {"bytes": io + sum(2 * row * n for n in lens) + 8 * sum(qs), "flops": sum(4 * c["heads"] * D * t * n for t, n in zip(qs, lens))}
    seen, read = 0, 0
    for t, n in zip(qs, lens):
        first = max(0, n - t - c["window"] + 1)       # first key that the window of the first query reaches
        read += n - first + min(c["sinks"], first)
        for i in range(n - t, n):
            lo = max(0, i - c["window"] + 1)
            seen += i + 1 - lo + min(c["sinks"], lo)
    return {"bytes": io + 2 * row * read, "flops": 4 * c["heads"] * D * seen}


def prepare(c, seed):
    """A pool whose rows hold their tokens in shuffled pages, and what the call gets."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    P, G, H, n, T = c["page"], c["kv_heads"], c["heads"], c["n"], c["T"]
    lens = _lens(c)
    branch = c["op"] in ("fork", "compact")          # rows that the call fills follow the rows that hold tokens
    extra = 0
    if c["op"] == "fork":
        extra = n * (_ceil(T, P) + 2)
    elif c["op"] == "compact":
        extra = n * _ceil(c["budget"] + c["window"], P)
    held = [_ceil(x, P) for x in lens]
    n_pages = sum(held) + extra + 8
    max_pages = max(held) + _ceil(T, P) + 1
    n_rows = len(lens) + (n if branch else 0)
    order = torch.randperm(n_pages, generator=g, device=DEV)[:sum(held)].to(torch.int32).cpu()
    table = torch.zeros((n_rows, max_pages), dtype=torch.int32)
    at = 0
    for i, m in enumerate(held):
        table[i, :m] = order[at:at + m]
        at += m
    refs = torch.zeros(n_pages, dtype=torch.int32)
    refs[order.long()] = 1
    length = torch.zeros(n_rows, dtype=torch.int32)
    length[:len(lens)] = torch.tensor(lens, dtype=torch.int32)
    s = dict(case=c, table=table.to(DEV), refs=refs.to(DEV), len=length.to(DEV), page=P)
    for name in ("k", "v"):
        s[name] = torch.empty((c["layers"], n_pages, G, P, D), dtype=torch.bfloat16, device=DEV)
        for x in s[name]:
            x.copy_(torch.randn(x.shape, generator=g, device=DEV, dtype=torch.float32))
    made = lambda *shape: torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16)  # noqa: E731
    if branch:
        s["dst"] = torch.arange(len(lens), n_rows, dtype=torch.int32, device=DEV)
        s["src"] = (torch.arange(n, device=DEV) % len(lens)).to(torch.int32)
        s["n_new"] = torch.full((n,), T, dtype=torch.int32, device=DEV)
    else:
        s["rows"] = torch.randperm(n_rows, generator=g, device=DEV).to(torch.int32)
        s["n_tokens"] = torch.tensor(_queries(c), dtype=torch.int32, device=DEV)[s["rows"].long()]
    if c["op"] == "compact":
        sets = G if c["per_head"] else 1
        s["idx"] = torch.empty((n, c["layers"], sets, c["budget"]), dtype=torch.int32, device=DEV)
        for i, x in enumerate(lens):
            keep = torch.rand((c["layers"], sets, x - c["window"]), generator=g, device=DEV).argsort(-1)[..., :c["budget"]]
            s["idx"][i] = keep.sort(-1).values
        s["meta"] = torch.randint(-2**31, 2**31, (n, max(lens)), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
        s["meta_out"] = torch.zeros((n, c["layers"], sets, c["budget"] + c["window"]), dtype=torch.int32, device=DEV)
    if c["op"] == "move":
        # new tokens come out of a model token-major, all KV heads of a token together
        s["k_new"], s["v_new"] = made(n, c["layers"], T, G, D), made(n, c["layers"], T, G, D)
        if c["load"]:     # and the scoring passes read them head-major
            s["k_back"] = torch.zeros((n, c["layers"], G, T, D), dtype=torch.bfloat16, device=DEV)
            s["v_back"] = torch.zeros_like(s["k_back"])
    if c["op"] in ("tree", "sink"):
        u = torch.randn((G, D), generator=g, device=DEV)
        u = u / u.norm(dim=-1, keepdim=True)
        first = s["k"][:, s["table"][:, 0].long(), :, :4].float() + 6.0 * u[:, None]
        s["k"][:, s["table"][:, 0].long(), :, :4] = first.to(torch.bfloat16)
        q = torch.randn((n, T, H, D), generator=g, device=DEV) + 8.0 * u.repeat_interleave(H // G, 0)
        s["q"] = q.to(torch.bfloat16)
        s["o"] = torch.zeros((n, T, H, D), dtype=torch.bfloat16, device=DEV)
        s["lse"] = torch.zeros((n, T, H), dtype=torch.float32, device=DEV)
    if c["op"] == "tree":
        parent = torch.rand((n, T), generator=g, device=DEV).cpu()
        mask = torch.zeros((n, T), dtype=torch.int64)
        for j in range(T):     # a drafted token sees its parent's tokens and itself; a root sees the cache only
            up = (parent[:, j] * (j + 1)).long() - 1
            seen = torch.where(up >= 0, mask.gather(1, up.clamp(min=0)[:, None])[:, 0], torch.zeros(n, dtype=torch.int64))
            mask[:, j] = seen | (1 << j if j < 63 else -(1 << 63))
        s["mask"] = mask.to(DEV)
    if own:
        from paper_2606_01790_gb300 import starkv as sk
        w = c.get("window", 32) if c["op"] == "compact" else 1
        s["st"] = sk.init_state(sk.Config(n_layers=c["layers"], n_heads=H, n_kv_heads=G, window=w, max_seqs=n,
                                         select_mode=int(c.get("per_head", False))))
        s["pages"] = sk.Pages(k=s["k"], v=s["v"], table=s["table"], len=s["len"], refs=s["refs"])
        s["ws"] = sk.pages_workspace(s["st"], s["pages"], n, T)
    return s


def run(s):
    return {"fork": _fork, "compact": _compact, "move": _move, "tree": _attend, "sink": _attend}[s["case"]["op"]](s)


def _words(x):
    return x.view(torch.int16)


def _fork(s):
    c = s["case"]
    if own:
        from paper_2606_01790_gb300 import starkv as sk
        st, pages = s["st"], s["pages"]
        sk.pages_free(st, pages, s["dst"])
        sk.pages_fork(st, pages, s["src"], s["dst"], s["ws"])
        sk.pages_extend(st, pages, s["dst"], s["n_new"], s["ws"])
    else:
        _plain_free(s, s["dst"].long())
        _plain_fork(s, s["src"].long(), s["dst"].long())
        _plain_extend(s, s["dst"].long(), s["n_new"].long(), c["T"])
    return {"table": s["table"], "len": s["len"], "refs": s["refs"], "k": _words(s["k"]), "v": _words(s["v"])}


def _compact(s):
    c = s["case"]
    if own:
        from paper_2606_01790_gb300 import starkv as sk
        st, pages = s["st"], s["pages"]
        sk.pages_free(st, pages, s["dst"])
        sk.pages_fork(st, pages, s["src"], s["dst"], s["ws"])
        seqs = [sk.Seq(L=x, budget=c["budget"], slot=i, idx=s["idx"][i], meta=s["meta"][i], meta_out=s["meta_out"][i])
                for i, x in enumerate(_lens(c))]
        sk.pages_compact(st, pages, s["dst"], seqs, s["ws"])
    else:
        _plain_free(s, s["dst"].long())
        _plain_fork(s, s["src"].long(), s["dst"].long())
        _plain_compact(s, s["dst"].long())
    return {"table": s["table"], "len": s["len"], "refs": s["refs"], "k": _words(s["k"]), "v": _words(s["v"]),
            "meta": s["meta_out"]}


def _move(s):
    c = s["case"]
    if own:
        from paper_2606_01790_gb300 import starkv as sk
        st, pages = s["st"], s["pages"]
        new = sk.Tokens(k=s["k_new"], v=s["v_new"], rows=s["rows"], n_tokens=s["n_tokens"])
        sk.pages_store(st, pages, 0, new)
        if c["load"]:
            back = sk.Tokens(k=s["k_back"].transpose(2, 3), v=s["v_back"].transpose(2, 3), rows=s["rows"],
                             n_tokens=s["n_tokens"])
            sk.pages_load(st, pages, 0, back)
    else:
        page, slot, take, valid = _places(s, c["T"])
        seq = torch.arange(c["n"], device=DEV)[:, None]
        for name in ("k", "v"):
            x = s[name]
            x[:, page, :, slot] = s[name + "_new"].transpose(1, 2)[seq, take]       # [n, T, layers, G, D]
            if c["load"]:
                got = x[:, page, :, slot].permute(0, 2, 3, 1, 4)
                s[name + "_back"].copy_(torch.where(valid[:, None, None, :, None], got, s[name + "_back"]))
    out = {"k": _words(s["k"]), "v": _words(s["v"])}
    if c["load"]:
        out.update(k_back=_words(s["k_back"]), v_back=_words(s["v_back"]))
    return out


def _attend(s):
    c = s["case"]
    if own:
        from paper_2606_01790_gb300 import starkv as sk
        qs = sk.Queries(q=s["q"], o=s["o"], lse=s["lse"], rows=s["rows"], n_tokens=s["n_tokens"], mask=s.get("mask"))
        if c["op"] == "tree":
            sk.tree_attention(s["st"], s["pages"], 1, qs, s["ws"])
        else:
            sk.sink_attention(s["st"], s["pages"], 1, qs, c["sinks"], c["window"], s["ws"])
        return {"o": s["o"], "lse": s["lse"]}
    return _plain_attend(s)


# ---------------------------------------------------------------- the plain forms

def _held(s, rows):
    """Pages of some rows: their numbers, and which entries of the table are theirs."""
    pages = (s["len"][rows].long() + s["page"] - 1) // s["page"]
    at = torch.arange(s["table"].shape[1], device=DEV)
    return s["table"][rows].long(), at < pages[:, None], pages


def _count(s, ids, theirs, sign):
    ones = torch.where(theirs, sign, 0).to(torch.int32)
    s["refs"].scatter_add_(0, torch.where(theirs, ids, 0).reshape(-1), ones.reshape(-1))


def _plain_free(s, rows):
    ids, theirs, _ = _held(s, rows)
    _count(s, ids, theirs, -1)
    s["len"][rows] = 0


def _plain_fork(s, src, dst):
    ids, theirs, _ = _held(s, src)
    _count(s, ids, theirs, 1)
    s["table"][dst] = torch.where(theirs, ids, s["table"][dst].long()).to(torch.int32)
    s["len"][dst] = s["len"][src]


def _taken(s, need, most):
    """The lowest free pages, `need` of them for each row in turn: [rows, most], and which of them count."""
    free = torch.argsort((s["refs"] != 0).to(torch.int32), stable=True)
    j = torch.arange(most, device=DEV)
    theirs = j < need[:, None]
    place = (need.cumsum(0) - need)[:, None] + j
    return free[torch.where(theirs, place, 0)], theirs


def _plain_extend(s, rows, n_new, most_new):
    P, length = s["page"], s["len"][rows].long()
    ids, _, held = _held(s, rows)
    last = ids.gather(1, (held - 1).clamp(min=0)[:, None])[:, 0]
    fill = length % P
    copy = (fill > 0) & (s["refs"][last] > 1)          # a shared last page is copied before it is appended to
    need = (length + n_new + P - 1) // P - held + copy
    new, theirs = _taken(s, need, most_new // P + 2)
    _count(s, new, theirs, 1)
    _count(s, last, copy, -1)
    at = (held - copy.long())[:, None] + torch.arange(new.shape[1], device=DEV)
    at = at.clamp(max=s["table"].shape[1] - 1)
    whole = s["table"][rows].long()
    # entries that do not count write back what stands at the last entry, which no row of these cases uses
    at = torch.where(theirs, at, s["table"].shape[1] - 1)
    s["table"][rows] = whole.scatter(1, at, torch.where(theirs, new, whole[:, -1:])).to(torch.int32)
    target = torch.where(copy, new[:, 0], last)
    kept = (torch.arange(P, device=DEV) < fill[:, None]) & copy[:, None]
    for x in (s["k"], s["v"]):
        x[:, target] = torch.where(kept[None, :, None, :, None], x[:, last], x[:, target])
    s["len"][rows] = (length + n_new).to(torch.int32)


def _plain_compact(s, rows):
    c, P = s["case"], s["page"]
    kept = c["budget"] + c["window"]
    ids, theirs, _ = _held(s, rows)
    need = torch.full((c["n"],), _ceil(kept, P), device=DEV)
    new, every = _taken(s, need, _ceil(kept, P))
    G = c["kv_heads"]
    layer = torch.arange(c["layers"], device=DEV)[:, None, None]
    head = torch.arange(G, device=DEV)[None, :, None]
    to = torch.arange(kept, device=DEV)
    window = s["len"][rows].long()[:, None] - c["window"] + torch.arange(c["window"], device=DEV)
    window = window[:, None, None].expand(-1, *s["idx"].shape[1:3], -1)
    at = torch.cat((s["idx"].long(), window), -1)              # [n, layers, sets, kept]: the tokens that stay
    page = ids.gather(1, (at // P).flatten(1)).view_as(at)
    for x in (s["k"], s["v"]):
        x[layer, new[:, to // P][:, None, None], head, to % P] = x[layer, page, head, at % P]
    s["meta_out"].copy_(s["meta"].gather(1, at.flatten(1)).view_as(at))
    _count(s, new, every, 1)
    _count(s, ids, theirs, -1)
    s["table"][rows, :new.shape[1]] = new.to(torch.int32)
    s["len"][rows] = kept


def _places(s, T):
    """Of each row's last n_tokens tokens, [n, T]: page, slot, number in the call, and which of them count;
    the places that do not are the row's last."""
    rows, count = s["rows"].long(), s["n_tokens"].long()
    t = torch.arange(T, device=DEV)
    take = torch.minimum(t[None], count[:, None] - 1)
    at = (s["len"][rows].long() - count)[:, None] + take
    return s["table"][rows].long().gather(1, at // s["page"]), at % s["page"], take, t < count[:, None]


def _plain_attend(s):
    c = s["case"]
    G, H, T = c["kv_heads"], c["heads"], c["T"]
    rows, count, length = s["rows"].long(), s["n_tokens"].long(), s["len"][s["rows"].long()].long()
    pages = max(_ceil(x, s["page"]) for x in _lens(c))
    ids = s["table"][rows, :pages].long()
    at = torch.arange(pages * s["page"], device=DEV)
    held = at < length[:, None]
    k, v = (x[1][torch.where(at[::s["page"]] < length[:, None], ids, 0)].transpose(1, 2).flatten(2, 3).float() for x in (s["k"], s["v"]))
    v = torch.where(held[:, None, :, None], v, 0.0)
    place = (length - count)[:, None] + torch.arange(T, device=DEV)      # position of each query
    if c["op"] == "tree":
        drafted = at - (length - count)[:, None]
        bit = (s["mask"][..., None] >> drafted.clamp(0, 63)[:, None]) & 1
        seen = (drafted < 0)[:, None] | ((bit == 1) & (drafted < count[:, None])[:, None])
    else:
        seen = (at <= place[..., None]) & ((at < c["sinks"]) | (at > place[..., None] - c["window"]))
    seen = (seen & held[:, None])[:, None, :, None]          # [n, 1, T, 1, keys]
    q = s["q"].float().view(c["n"], T, G, H // G, D).transpose(1, 2)
    z = (q.flatten(2, 3) @ k.transpose(2, 3)).view(c["n"], G, T, H // G, -1) / math.sqrt(D)
    z = torch.where(seen, z, -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    p = torch.exp(z - top)
    total = p.sum(-1, keepdim=True)
    o = (p.flatten(2, 3) @ v).view(c["n"], G, T, H // G, D) / torch.where(total > 0, total, 1.0)
    lse = (torch.log(total) + top)[..., 0]
    real = torch.arange(T, device=DEV) < count[:, None]
    o = o.transpose(1, 2).reshape(c["n"], T, H, D).to(torch.bfloat16)
    lse = lse.transpose(1, 2).reshape(c["n"], T, H)
    return {"o": torch.where(real[..., None, None], o, s["o"]), "lse": torch.where(real[..., None], lse, s["lse"])}


# ---------------------------------------------------------------- from the definition, in 64 bits

def exact(c, seed):
    """The attention of each query over the keys that it sees, one row and one KV head at a time, in 64 bits;
    nothing for the operators that copy and count."""
    if c["op"] not in ("tree", "sink"):
        return None
    s = prepare(c, seed)
    H, G, P = c["heads"], c["kv_heads"], c["page"]
    o = torch.zeros((c["n"], c["T"], H, D), dtype=torch.float64, device=DEV)
    lse = torch.zeros((c["n"], c["T"], H), dtype=torch.float64, device=DEV)
    rows, counts, lengths = s["rows"].tolist(), s["n_tokens"].tolist(), s["len"].tolist()
    for i, (r, T) in enumerate(zip(rows, counts)):
        L = lengths[r]
        pages = s["table"][r, :_ceil(L, P)].long()
        bias = torch.full((T, L), -math.inf, dtype=torch.float64, device=DEV)
        if c["op"] == "tree":
            bias[:, :L - T] = 0
            bits = torch.tensor([[(m >> j) & 1 for j in range(T)] for m in s["mask"][i, :T].tolist()], device=DEV)
            bias[:, L - T:][bits == 1] = 0
        else:
            for t in range(T):
                p = L - T + t
                bias[t, max(0, p - c["window"] + 1):p + 1] = 0
                bias[t, :min(c["sinks"], p + 1)] = 0
        for g in range(G):
            keys = s["k"][1, pages, g].reshape(-1, D)[:L].double()
            values = s["v"][1, pages, g].reshape(-1, D)[:L].double()
            for h in range(g * (H // G), (g + 1) * (H // G)):
                z = s["q"][i, :T, h].double() @ keys.T / math.sqrt(D) + bias
                lse[i, :T, h] = torch.logsumexp(z, -1)
                o[i, :T, h] = torch.softmax(z, -1) @ values
    return {"o": o, "lse": lse}
