"""What eviction by attention weight and attention over chosen pages are measured on.

A case is one pass of an operator of the paged cache (pages of ``page`` tokens
that the rows of a page table hold, every layer of a token under one page number):

* ``mass``    the attention weights that new tokens give to each cached token are
              added to what it has had so far, per KV head: after an attention with
              a sliding window and sinks, or of drafted tokens (``tree``), whose
              normalisers are at hand;
* ``evict``   a branch of each row keeps the tokens with the greatest mass and its
              recent window, in pages of its own, and their mass with them;
* ``bounds``  per page, KV head and channel the least and the greatest key, for the
              pages that hold the last tokens of each row;
* ``sparse``  each query scores the pages by these bounds, takes the best, the first
              and the last ones, and attends over the tokens that they hold.

The shapes are the repository's workloads (28 query and 4 KV heads, or 32 and 8;
caches of 5 and 20 screenshots before and after their compression; batches of ragged
lengths) with pages of 16 to 128 tokens in shuffled order.  Keys, values and queries
are normal; the keys of a page share a direction of their own, the first four keys
and all queries another, so that some pages and the first tokens take more of the
attention, as they do in real caches.  What is copied is compared as 16-bit words.
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
        # the smallest call: one new token of a short cache
        _case("mass_tiny", "mass", ctx=577, tree=False, sinks=4, window=512, decay=1.0),
        # serving: one layer's new token of 64 rows of many lengths, older weights fading
        _case("mass_decode_64", "mass", n=64, ctx=14033, ragged=True, page=32, heads=32, kv_heads=8, tree=False, sinks=0,
              window=1 << 20, decay=0.98),
        # serving: 32 rows of many lengths, 26 drafted tokens each
        _case("mass_tree_32", "mass", n=32, ctx=14033, ragged=True, T=26, tree=True, decay=1.0),
        # one screenshot's tokens appended at once
        _case("mass_chunk", "mass", ctx=8113, T=2704, tree=False, sinks=64, window=4096, decay=0.9),
        # one step's eviction of a five-screenshot cache: every KV head keeps 2704 tokens of its own and the window
        _case("evict_5shot", "evict", layers=28, ctx=14032, budget=2704, window=32, per_head=True),
        # eight trajectories of many lengths, one set of tokens for all KV heads
        _case("evict_ragged_8", "evict", layers=28, n=8, ctx=12001, ragged=True, page=16, budget=2048, window=32,
              per_head=False),
        # serving: the new token of 64 rows, every layer
        _case("bounds_decode_64", "bounds", layers=28, n=64, ctx=14033, ragged=True, page=32, heads=32, kv_heads=8),
        # a five-screenshot cache has just been stored
        _case("bounds_prompt", "bounds", layers=28, ctx=14032, T=14032),
        # one token over a compressed cache
        _case("sparse_first", "sparse", ctx=2737, first=1, last=2, chosen=16),
        # serving: 64 rows of many lengths, one token each
        _case("sparse_decode_64", "sparse", n=64, ctx=14033, ragged=True, page=32, heads=32, kv_heads=8, first=1, last=4,
              chosen=64),
        # four 20-screenshot caches, one token each
        _case("sparse_long", "sparse", n=4, ctx=56193, first=1, last=4, chosen=128),
        # four rows, eight drafted tokens in a line, each with pages of its own
        _case("sparse_draft", "sparse", n=4, ctx=14041, ragged=True, T=8, first=1, last=2, chosen=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["mass", "mass", "evict", "bounds", "sparse", "sparse"])
    heads, kv_heads = rng.choice([(28, 4), (28, 4), (32, 8), (16, 2), (8, 8), (40, 8), (12, 1)])
    c = _case("", op, heads=heads, kv_heads=kv_heads, page=rng.choice([16, 32, 64, 64, 128]),
              ctx=_log(rng, 600, 14000), ragged=rng.random() < 0.6)
    del c["name"]
    if op == "mass":
        c.update(n=_log(rng, 1, 64), tree=rng.random() < 0.4, decay=rng.choice([1.0, 0.9, 0.98, 0.5]))
        if c["tree"]:
            c.update(T=rng.randint(1, 64))
        else:
            c.update(T=rng.choice([1, 1, _log(rng, 2, 600)]), sinks=rng.choice([0, 1, 4, 64]), window=_log(rng, 64, 16384))
    elif op == "evict":
        c.update(layers=_log(rng, 1, 28), n=_log(rng, 1, 8), window=rng.choice([8, 16, 32]), per_head=rng.random() < 0.5)
        while heads // kv_heads * c["window"] > 256:
            c["window"] //= 2
        c["budget"] = _log(rng, 50, max(51, c["ctx"] // 2))
    elif op == "bounds":
        c.update(layers=_log(rng, 1, 28), n=_log(rng, 1, 64))
        c["T"] = rng.choice([1, 1, _log(rng, 1, c["ctx"])])
    else:
        c.update(n=_log(rng, 1, 64), T=rng.choice([1, 1, _log(rng, 2, 64)]), first=rng.choice([0, 1, 2]), last=rng.randint(1, 4))
        c["chosen"] = c["first"] + c["last"] + _log(rng, 1, 128)
    while c["n"] > 1 and _cost(c) > _MOST[op]:
        c["n"] -= 1
    while c["T"] > 1 and _cost(c) > _MOST[op]:
        c["T"] = c["T"] // 2
    return c


def _cost(c):
    w = work(dict(c, name=""))
    each = 0      # bytes of K and V that the queries take one by one
    if c["op"] == "sparse":
        each = c["n"] * c["T"] * min(c["ctx"], c["chosen"] * c["page"]) * c["kv_heads"] * D * 4
    return max(w["bytes"], w["flops"] / 50, each / 4)


_MOST = dict(mass=1.5e9, evict=1e9, bounds=420e6, sparse=600e6)


def _lens(c):
    """Tokens of each row before the call: they depend on the case alone.  A row is at least a quarter
    of the longest, and long enough for the call."""
    rng = random.Random(c["ctx"] * 131 + c["n"])
    least = c["budget"] + c["window"] if c["op"] == "evict" else c["T"]
    return [max(least, rng.randint(c["ctx"] // 4, c["ctx"]) if c["ragged"] and i else c["ctx"]) for i in range(c["n"])]


def _queries(c):
    """Real queries (new tokens) of each row: all T, or fewer behind the first of a ragged batch."""
    rng = random.Random(c["T"] * 17 + c["n"])
    return [rng.randint(max(1, c["T"] // 2), c["T"]) if c["ragged"] and i else c["T"] for i in range(c["n"])]


def _ceil(a, b):
    return -(-a // b)


def work(c):
    row = c["kv_heads"] * D * 2      # bytes of one token's K (or V) in a layer
    H, G, P = c["heads"], c["kv_heads"], c["page"]
    lens, qs = _lens(c), _queries(c)
    if c["op"] == "evict":
        sets = G if c["per_head"] else 1
        kept = c["budget"] + c["window"]
        b = c["n"] * c["layers"] * (4 * kept * row + 4 * sets * c["budget"] + 8 * sets * kept + 4 * G * kept)
        b += sum(4 * G * c["layers"] * n + 4 * 4 * (_ceil(n, P) + _ceil(kept, P)) for n in lens)
        return {"bytes": b, "flops": 0}
    if c["op"] == "bounds":
        b = 0
        for t, n in zip(qs, lens):
            first = (n - t) // P
            b += c["layers"] * ((n - first * P) * row + (_ceil(n, P) - first) * 2 * row)
        return {"bytes": b, "flops": 0}
    if c["op"] == "sparse":
        b = f = 0
        for t, n in zip(qs, lens):
            pages = _ceil(n, P)
            b += pages * 2 * row + 2 * row * min(n, t * c["chosen"] * P) + t * (H * (4 * D + 4) + 4 * G * c["chosen"])
            f += t * (4 * G * D * pages + 4 * H * D * min(n, c["chosen"] * P))
        return {"bytes": b, "flops": f}
    b = f = 0
    for t, n in zip(qs, lens):
        if c["tree"]:
            seen, read = t * (n - t) + t * t // 2, n
        else:
            seen, first = 0, max(0, n - t - c["window"] + 1)       # first key that the window of the first query reaches
            read = n - first + min(c["sinks"], first)
            for i in range(n - t, n):
                lo = max(0, i - c["window"] + 1)
                seen += i + 1 - lo + min(c["sinks"], lo)
        b += t * H * (2 * D + 4) + read * row + 8 * G * (n if c["decay"] != 1.0 else read)
        f += 2 * H * D * seen
    return {"bytes": b, "flops": f}


def prepare(c, seed):
    """A pool whose rows hold their tokens in shuffled pages, and what the call gets."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    P, G, H, n, T = c["page"], c["kv_heads"], c["heads"], c["n"], c["T"]
    lens, evict = _lens(c), c["op"] == "evict"          # (an eviction works on branches, in rows behind the others)
    held = [_ceil(x, P) for x in lens]
    n_pages = sum(held) + 8 + (n * _ceil(c["budget"] + c["window"], P) if evict else 0)
    max_pages = max(held) + 1
    n_rows = n * (2 if evict else 1)
    order = torch.randperm(n_pages, generator=g, device=DEV)[:sum(held)].to(torch.int32).cpu()
    table = torch.zeros((n_rows, max_pages), dtype=torch.int32)
    at = 0
    for i, m in enumerate(held):
        table[i, :m] = order[at:at + m]
        at += m
    refs = torch.zeros(n_pages, dtype=torch.int32)
    refs[order.long()] = 1
    length = torch.zeros(n_rows, dtype=torch.int32)
    length[:n] = torch.tensor(lens, dtype=torch.int32)
    s = dict(case=c, table=table.to(DEV), refs=refs.to(DEV), len=length.to(DEV), page=P)
    for name in ("k", "v"):
        s[name] = torch.empty((c["layers"], n_pages, G, P, D), dtype=torch.bfloat16, device=DEV)
        for x in s[name]:
            x.copy_(torch.randn(x.shape, generator=g, device=DEV, dtype=torch.float32))
            if name == "k":
                x.add_(0.5 * torch.randn((n_pages, G, 1, D), generator=g, device=DEV))
    u = torch.randn((G, D), generator=g, device=DEV)
    u = u / u.norm(dim=-1, keepdim=True)
    first = s["k"][:, s["table"][:n, 0].long(), :, :4].float() + 6.0 * u[:, None]
    s["k"][:, s["table"][:n, 0].long(), :, :4] = first.to(torch.bfloat16)
    if evict:
        s["src"] = torch.arange(n, dtype=torch.int32, device=DEV)
        s["dst"] = s["src"] + n
        sets = G if c["per_head"] else 1
        s["idx"] = torch.empty((n, c["layers"], sets, c["budget"]), dtype=torch.int32, device=DEV)
        s["meta"] = torch.randint(-2**31, 2**31, (n, max(lens)), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
        s["meta_out"] = torch.zeros((n, c["layers"], sets, c["budget"] + c["window"]), dtype=torch.int32, device=DEV)
    else:
        s["rows"] = torch.randperm(n_rows, generator=g, device=DEV).to(torch.int32)
        s["n_tokens"] = torch.tensor(_queries(c), dtype=torch.int32, device=DEV)[s["rows"].long()]
    if c["op"] in ("mass", "evict"):     # weights that tokens have had so far: a few have had most
        s["mass"] = torch.exp(1.5 * torch.randn((c["layers"], n_rows, G, max_pages * P), generator=g, device=DEV))
    if c["op"] in ("bounds", "sparse"):
        s["bounds"] = torch.randn((c["layers"], n_pages, G, 2, D), generator=g, device=DEV).to(torch.bfloat16)
    if c["op"] in ("mass", "sparse"):
        q = torch.randn((n, T, H, D), generator=g, device=DEV) + 4.0 * u.repeat_interleave(H // G, 0)
        s["q"] = q.to(torch.bfloat16)
        s["lse"] = torch.zeros((n, T, H), dtype=torch.float32, device=DEV)
    if c["op"] == "sparse":
        s["o"] = torch.zeros((n, T, H, D), dtype=torch.bfloat16, device=DEV)
        s["chosen"] = torch.full((n, T, G, c["chosen"]), -1, dtype=torch.int32, device=DEV)
        for r in range(n):               # the pages hold what an earlier call on them found
            ids = s["table"][r, :held[r]].long()
            fill = (lens[r] - P * torch.arange(held[r], device=DEV)).clamp(max=P)
            there = (torch.arange(P, device=DEV) < fill[:, None])[:, None, :, None]
            k = s["k"][:, ids].float()
            s["bounds"][:, ids, :, 0] = torch.where(there, k, math.inf).amin(3).to(torch.bfloat16)
            s["bounds"][:, ids, :, 1] = torch.where(there, k, -math.inf).amax(3).to(torch.bfloat16)
    if c["op"] == "mass":
        if c["tree"]:
            parent = torch.rand((n, T), generator=g, device=DEV).cpu()
            mask = torch.zeros((n, T), dtype=torch.int64)
            for j in range(T):     # a drafted token sees its parent's tokens and itself; a root sees the cache only
                up = (parent[:, j] * (j + 1)).long() - 1
                seen = torch.where(up >= 0, mask.gather(1, up.clamp(min=0)[:, None])[:, 0], torch.zeros(n, dtype=torch.int64))
                mask[:, j] = seen | (1 << j if j < 63 else -(1 << 63))
            s["mask"] = mask.to(DEV)
        z, _ = _plain_logits(s)
        s["lse"].copy_(torch.logsumexp(z, -1).transpose(1, 2).reshape(n, T, H))
        del z
    if own:
        from paper_2606_01790_gb300 import starkv as sk
        w = c["window"] if evict else 1
        s["st"] = sk.init_state(sk.Config(n_layers=c["layers"], n_heads=H, n_kv_heads=G, window=w, max_seqs=n,
                                         select_mode=int(c.get("per_head", False))))
        s["pages"] = sk.Pages(k=s["k"], v=s["v"], table=s["table"], len=s["len"], refs=s["refs"])
        if c["op"] == "sparse":
            s["ws"] = sk.sparse_workspace(s["st"], s["pages"], n, T, c["chosen"])
        else:
            s["ws"] = sk.pages_workspace(s["st"], s["pages"], n, T)
    return s


def run(s):
    return {"mass": _mass, "evict": _evict, "bounds": _bounds, "sparse": _sparse}[s["case"]["op"]](s)


def _words(x):
    return x.view(torch.int16)


def _mass(s):
    c = s["case"]
    if own:
        from paper_2606_01790_gb300 import starkv as sk
        qs = sk.Queries(q=s["q"], o=None, lse=s["lse"], rows=s["rows"], n_tokens=s["n_tokens"], mask=s.get("mask"))
        mass = sk.Mass(s["mass"], decay=c["decay"])
        if c["tree"]:
            sk.tree_mass(s["st"], s["pages"], 1, qs, mass, s["ws"])
        else:
            sk.sink_mass(s["st"], s["pages"], 1, qs, c["sinks"], c["window"], mass, s["ws"])
    else:
        _plain_mass(s)
    return {"mass": s["mass"]}


def _evict(s):
    c = s["case"]
    if own:
        from paper_2606_01790_gb300 import starkv as sk
        st, pages = s["st"], s["pages"]
        sk.pages_free(st, pages, s["dst"])
        sk.pages_fork(st, pages, s["src"], s["dst"], s["ws"])
        s["mass"][:, c["n"]:] = s["mass"][:, :c["n"]]
        seqs = [sk.Seq(L=x, budget=c["budget"], slot=i, idx=s["idx"][i], meta=s["meta"][i], meta_out=s["meta_out"][i])
                for i, x in enumerate(_lens(c))]
        sk.pages_evict(st, pages, s["dst"], seqs, sk.Mass(s["mass"]), s["ws"])
    else:
        _plain_evict(s)
    return {"table": s["table"], "len": s["len"], "refs": s["refs"], "k": _words(s["k"]), "v": _words(s["v"]),
            "meta": s["meta_out"], "idx": s["idx"], "mass": s["mass"]}


def _bounds(s):
    c = s["case"]
    if own:
        from paper_2606_01790_gb300 import starkv as sk
        sk.pages_bounds(s["st"], s["pages"], 0, c["layers"], s["bounds"], c["T"], rows=s["rows"], n_tokens=s["n_tokens"])
    else:
        _plain_bounds(s)
    return {"bounds": s["bounds"]}


def _sparse(s):
    c = s["case"]
    if own:
        from paper_2606_01790_gb300 import starkv as sk
        qs = sk.Queries(q=s["q"], o=s["o"], lse=s["lse"], rows=s["rows"], n_tokens=s["n_tokens"])
        sk.sparse_attention(s["st"], s["pages"], 1, qs, s["bounds"], c["first"], c["last"], c["chosen"], s["ws"],
                            chosen_out=s["chosen"])
        return {"o": s["o"], "lse": s["lse"], "chosen": s["chosen"]}
    return _plain_sparse(s)


# ---------------------------------------------------------------- the plain forms

def _plain_logits(s):
    """Logits of the queries over every key of their rows, -inf where not seen: [n, G, T, heads of a group, keys];
    and which queries are real."""
    c = s["case"]
    G, H, T = c["kv_heads"], c["heads"], c["T"]
    rows, count, length = s["rows"].long(), s["n_tokens"].long(), s["len"][s["rows"].long()].long()
    pages = max(_ceil(x, s["page"]) for x in _lens(c))
    ids = s["table"][rows, :pages].long()
    at = torch.arange(pages * s["page"], device=DEV)
    held = at < length[:, None]
    k = s["k"][1][torch.where(at[::s["page"]] < length[:, None], ids, 0)].transpose(1, 2).flatten(2, 3).float()
    place = (length - count)[:, None] + torch.arange(T, device=DEV)      # position of each query
    if c["tree"]:
        drafted = at - (length - count)[:, None]
        bit = (s["mask"][..., None] >> drafted.clamp(0, 63)[:, None]) & 1
        seen = (drafted < 0)[:, None] | ((bit == 1) & (drafted < count[:, None])[:, None])
    else:
        seen = (at <= place[..., None]) & ((at < c["sinks"]) | (at > place[..., None] - c["window"]))
    real = torch.arange(T, device=DEV) < count[:, None]
    seen = (seen & held[:, None] & real[..., None])[:, None, :, None]          # [n, 1, T, 1, keys]
    q = s["q"].float().view(c["n"], T, G, H // G, D).transpose(1, 2)
    z = (q.flatten(2, 3) @ k.transpose(2, 3)).view(c["n"], G, T, H // G, -1) / math.sqrt(D)
    return torch.where(seen, z, -math.inf), real


def _plain_mass(s):
    c = s["case"]
    G, T, n = c["kv_heads"], c["T"], c["n"]
    z, real = _plain_logits(s)
    lse = s["lse"].view(n, T, G, -1).transpose(1, 2)
    lse = torch.where(real[:, None, :, None], lse, 0.0)
    new = torch.exp(z - lse[..., None]).flatten(2, 3).sum(2)          # [n, G, keys]
    rows, count, length = s["rows"].long(), s["n_tokens"].long(), s["len"][s["rows"].long()].long()
    keys = new.shape[-1]
    at = torch.arange(keys, device=DEV)
    old = s["mass"][1, rows, :, :keys]
    fresh = (at >= (length - count)[:, None])[:, None]                # tokens of this call start at nothing
    made = torch.where(fresh, 0.0, old * c["decay"]) + new
    s["mass"][1, rows, :, :keys] = torch.where((at < length[:, None])[:, None], made, old)


def _held(s, rows):
    """Pages of some rows: their numbers, and which entries of the table are theirs."""
    pages = (s["len"][rows].long() + s["page"] - 1) // s["page"]
    at = torch.arange(s["table"].shape[1], device=DEV)
    return s["table"][rows].long(), at < pages[:, None]


def _count(s, ids, theirs, sign):
    ones = torch.where(theirs, sign, 0).to(torch.int32)
    s["refs"].scatter_add_(0, torch.where(theirs, ids, 0).reshape(-1), ones.reshape(-1))


def _plain_evict(s):
    c, P, G, n = s["case"], s["page"], s["case"]["kv_heads"], s["case"]["n"]
    src, dst = s["src"].long(), s["dst"].long()
    kept, w = c["budget"] + c["window"], c["window"]
    # the branches go, and come again
    _count(s, *_held(s, dst), -1)
    ids, theirs = _held(s, src)
    _count(s, ids, theirs, 1)
    s["table"][dst] = torch.where(theirs, ids, s["table"][dst].long()).to(torch.int32)
    s["len"][dst] = s["len"][src]
    s["mass"][:, n:] = s["mass"][:, :n]
    # the heaviest tokens before the window
    length = s["len"][dst].long()
    mass = s["mass"][:, dst].transpose(0, 1)                          # [n, layers, G, tokens]
    heavy = mass if c["per_head"] else mass.double().sum(2, keepdim=True)
    past = torch.arange(heavy.shape[-1], device=DEV) < (length - w)[:, None]
    heavy = torch.where(past[:, None, None], heavy, -math.inf)
    keep = torch.sort(heavy, dim=-1, descending=True, stable=True).indices[..., :c["budget"]].sort(-1).values
    s["idx"].copy_(keep)
    # in pages of their own
    window = (length - w)[:, None, None, None] + torch.arange(w, device=DEV)
    at = torch.cat((keep, window.expand(-1, *keep.shape[1:3], -1)), -1)   # [n, layers, sets, kept]
    free = torch.argsort((s["refs"] != 0).to(torch.int32), stable=True)
    new = free[:n * _ceil(kept, P)].view(n, -1)
    to = torch.arange(kept, device=DEV)
    layer = torch.arange(c["layers"], device=DEV)[:, None, None]
    head = torch.arange(G, device=DEV)[None, :, None]
    page = ids.gather(1, (at // P).flatten(1)).view_as(at)
    for x in (s["k"], s["v"]):
        x[layer, new[:, to // P][:, None, None], head, to % P] = x[layer, page, head, at % P]
    s["meta_out"].copy_(s["meta"].gather(1, at.flatten(1)).view_as(at))
    s["mass"][:, dst, :, :kept] = mass.gather(-1, at.expand(-1, -1, G, -1)).transpose(0, 1)
    _count(s, new, torch.ones_like(new, dtype=torch.bool), 1)
    _count(s, ids, theirs, -1)
    s["table"][dst, :new.shape[1]] = new.to(torch.int32)
    s["len"][dst] = kept


def _plain_bounds(s):
    c, P = s["case"], s["page"]
    rows, count = s["rows"].long(), s["n_tokens"].long()
    length = s["len"][rows].long()
    first, end = (length - count) // P, (length + P - 1) // P
    most = (c["T"] + P - 2) // P + 1
    at = first[:, None] + torch.arange(most, device=DEV)              # [n, most] pages of each row, in order
    seq, j = (at < end[:, None]).nonzero(as_tuple=True)
    at = at[seq, j]
    ids = s["table"][rows[seq], at].long()
    there = (torch.arange(P, device=DEV) < (length[seq] - at * P)[:, None])[:, None, :, None]
    k = s["k"][:, ids].float()
    s["bounds"][:, ids, :, 0] = torch.where(there, k, math.inf).amin(3).to(torch.bfloat16)
    s["bounds"][:, ids, :, 1] = torch.where(there, k, -math.inf).amax(3).to(torch.bfloat16)


def _plain_sparse(s):
    c, P = s["case"], s["page"]
    G, H, T, n = c["kv_heads"], c["heads"], c["T"], c["n"]
    rows, count, length = s["rows"].long(), s["n_tokens"].long(), s["len"][s["rows"].long()].long()
    pages = max(_ceil(x, P) for x in _lens(c))
    real = torch.arange(T, device=DEV) < count[:, None]
    place = torch.where(real, (length - count)[:, None] + torch.arange(T, device=DEV), 0)
    last = (place // P)[..., None]                                    # [n, T, 1]: the page that a query is in
    page = torch.arange(pages, device=DEV)
    ids = torch.where(page * P < length[:, None], s["table"][rows, :pages].long(), 0)
    # scores: the most that the logits of a page's keys can come to, added up over the heads of a group (in 64 bits:
    # which of two pages is taken hangs on the last bit)
    q = s["q"].double().view(n, T, G, H // G, D)
    up, down = q.clamp(min=0).sum(3).transpose(1, 2), q.clamp(max=0).sum(3).transpose(1, 2)      # [n, G, T, D]
    b = s["bounds"][1][ids].double().permute(0, 2, 3, 4, 1)          # [n, G, 2, D, pages]
    score = (up @ b[:, :, 1] + down @ b[:, :, 0]).transpose(1, 2)     # [n, T, G, pages]
    always = (page < c["first"]) | (page > last - c["last"])
    score = torch.where(always[:, :, None], math.inf, score)
    score = torch.where((page <= last)[:, :, None], score, -math.inf)
    most = min(c["chosen"], pages)
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :most]
    best = torch.where(best <= last[..., None], best, pages).sort(-1).values
    there = best < pages
    chosen = torch.where(there, best, -1)
    # attention over what they hold
    own_ids = ids[:, None, None].expand(-1, T, G, -1).gather(-1, best.clamp(max=pages - 1))
    head = torch.arange(G, device=DEV)[:, None]
    k, v = (x[1][own_ids, head].flatten(3, 4).float() for x in (s["k"], s["v"]))     # [n, T, G, keys, D]
    at = (best[..., None] * P + torch.arange(P, device=DEV)).flatten(3)
    seen = (at <= place[:, :, None, None])[:, :, :, None]
    v = torch.where(seen[..., 0, :, None], v, 0.0)
    z = (s["q"].float().view(n, T, G, H // G, D) @ k.transpose(3, 4)) / math.sqrt(D)
    z = torch.where(seen, z, -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - top)
    total = p.sum(-1, keepdim=True)
    o = ((p @ v) / total).reshape(n, T, H, D).to(torch.bfloat16)
    lse = (torch.log(total) + top).reshape(n, T, H)
    out = s["chosen"].clone()
    out[..., :most] = torch.where(real[..., None, None], chosen, out[..., :most]).to(torch.int32)
    return {"o": torch.where(real[..., None, None], o, s["o"]), "lse": torch.where(real[..., None], lse, s["lse"]), "chosen": out}


# ---------------------------------------------------------------- from the definition, in 64 bits

def exact(c, seed):
    """The definitions row by row and head by head in 64 bits; nothing for the operator that sorts and copies."""
    if c["op"] == "evict":
        return None
    s = prepare(c, seed)
    return {"mass": _exact_mass, "bounds": _exact_bounds, "sparse": _exact_sparse}[c["op"]](s)


def _exact_mass(s):
    c = s["case"]
    hg, P = c["heads"] // c["kv_heads"], c["page"]
    out = s["mass"].double()
    rows, counts, lengths = s["rows"].tolist(), s["n_tokens"].tolist(), s["len"].tolist()
    for i, (r, T) in enumerate(zip(rows, counts)):
        L = lengths[r]
        pages = s["table"][r, :_ceil(L, P)].long()
        seen = torch.zeros((T, L), dtype=torch.float64, device=DEV)
        if c["tree"]:
            seen[:, :L - T] = 1
            seen[:, L - T:] = torch.tensor([[(m >> j) & 1 for j in range(T)] for m in s["mask"][i, :T].tolist()], device=DEV)
        else:
            for t in range(T):
                p = L - T + t
                seen[t, max(0, p - c["window"] + 1):p + 1] = 1
                seen[t, :min(c["sinks"], p + 1)] = 1
        for g in range(c["kv_heads"]):
            keys = s["k"][1, pages, g].reshape(-1, D)[:L].double()
            had = out[1, r, g, :L] * c["decay"]
            had[L - T:] = 0
            for h in range(g * hg, (g + 1) * hg):
                z = s["q"][i, :T, h].double() @ keys.T / math.sqrt(D) - s["lse"][i, :T, h, None].double()
                had += (torch.exp(z) * seen).sum(0)
            out[1, r, g, :L] = had
    return {"mass": out}


def _exact_bounds(s):
    c, P = s["case"], s["page"]
    out = s["bounds"].double()
    for r, T in zip(s["rows"].tolist(), s["n_tokens"].tolist()):
        L = int(s["len"][r])
        for j in range((L - T) // P, _ceil(L, P)):
            page = int(s["table"][r, j])
            k = s["k"][:, page, :, :min(P, L - j * P)].double()
            out[:, page] = torch.stack((k.min(2).values, k.max(2).values), 2)
    return {"bounds": out}


def _exact_sparse(s):
    c, P = s["case"], s["page"]
    G, H = c["kv_heads"], c["heads"]
    hg = H // G
    o, lse, chosen = s["o"].double(), s["lse"].double(), s["chosen"].clone()
    rows, counts, lengths = s["rows"].tolist(), s["n_tokens"].tolist(), s["len"].tolist()
    for i, (r, T) in enumerate(zip(rows, counts)):
        pages = s["table"][r, :_ceil(lengths[r], P)].long()
        for g in range(G):
            least, most = s["bounds"][1, pages, g].double().unbind(1)
            keys, values = (x[1, pages, g].double() for x in (s["k"], s["v"]))
            for t in range(T):
                place = lengths[r] - T + t
                last = place // P
                q = s["q"][i, t, g * hg:(g + 1) * hg].double()
                score = torch.maximum(q[:, None] * least[:last + 1], q[:, None] * most[:last + 1]).sum((0, 2)).tolist()
                for j in range(last + 1):
                    if j < c["first"] or j > last - c["last"]:
                        score[j] = math.inf
                best = sorted(sorted(range(last + 1), key=lambda j: (-score[j], j))[:c["chosen"]])
                chosen[i, t, g, :len(best)] = torch.tensor(best, dtype=torch.int32)
                n_keys = (len(best) - 1) * P + place % P + 1
                z = q @ keys[best].reshape(-1, D)[:n_keys].T / math.sqrt(D)
                lse[i, t, g * hg:(g + 1) * hg] = torch.logsumexp(z, -1)
                o[i, t, g * hg:(g + 1) * hg] = torch.softmax(z, -1) @ values[best].reshape(-1, D)[:n_keys]
    return {"o": o, "lse": lse, "chosen": chosen}
