"""The operators on a paged key/value cache, as cases that can be timed: what a program does that lets the language
half of the model go on from a prefix - with text or action tokens, drafted several at a time - and keeps several
sequences at once.

  attend   pi0_tree_attention: the drafted tokens of every sequence (a tree given by bits, a chain, or one token each)
           against the sequence's pages and each other
  rope     pi0_qk_norm_rope: norm and rotation of the new tokens' queries and keys, keys and values into the pages
  pages    pi0_pages_fork, pi0_pages_compact and pi0_pages_reserve in a row: continuations forked off a sequence, some
           of its last tokens dropped, room made for the next draft (all layers of the cache)

Head layouts are the prefix transformer's own (8 query heads on one key/value head of 256) and generic grouped ones.
Lengths run from nothing to 16 thousand positions, drafts from one token to a few hundred.  `own` chooses between the
framework's entry points and the plain form below.
"""
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def attend(name, seqs, nodes, longest, heads, kv_heads, head_dim, page, dtype="bf16", ragged=True, tree="tree"):
    return {"name": name, "op": "attend", "seqs": seqs, "nodes": nodes, "longest": longest, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "page": page, "dtype": dtype, "ragged": ragged, "tree": tree}


def rope(name, seqs, nodes, longest, heads, kv_heads, head_dim, page, dtype="bf16", ragged=True, rope_dim=0, interleaved=False,
         tree="chain"):
    return {"name": name, "op": "rope", "seqs": seqs, "nodes": nodes, "longest": longest, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "page": page, "dtype": dtype, "ragged": ragged, "rope_dim": rope_dim or head_dim,
            "interleaved": interleaved, "tree": tree}


def pages(name, seqs, forks, longest, tail, tenths, extra, layers, kv_heads, head_dim, page, dtype="bf16"):
    return {"name": name, "op": "pages", "seqs": seqs, "forks": forks, "longest": longest, "tail": tail, "tenths": tenths,
            "extra": extra, "layers": layers, "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "dtype": dtype}


def listed():
    return [
        # one token after a prefix of three camera views and a full prompt: the smallest call, all latency
        attend("attend-1x1-816", 1, 1, 816, 8, 1, 256, 64, ragged=False, tree="chain"),
        # a full tree of drafts for one robot with a few thousand tokens of history
        attend("attend-tree-1x64-4k", 1, 64, 4096, 8, 1, 256, 64, ragged=False),
        # plain decoding of many sequences: the cache's bytes are all there is to it
        attend("attend-64x1-8k", 64, 1, 8192, 8, 1, 256, 64, tree="chain"),
        # small pages, grouped heads, odd drafts with rows that see nothing of the tree, a sequence without a past
        attend("attend-holes-16x33-3k", 16, 33, 3001, 16, 4, 128, 16, dtype="f16", tree="holes"),
        # many rows on long sequences: products instead of bytes
        attend("attend-tree-8x64-16k", 8, 64, 16384, 8, 1, 256, 64),
        # one token's heads
        rope("rope-1x1", 1, 1, 816, 8, 1, 256, 64, ragged=False),
        # trees of drafts: positions by depth, half of a head rotated, neighbours paired
        rope("rope-tree-16x33", 16, 33, 3001, 16, 4, 128, 16, dtype="f16", rope_dim=64, interleaved=True, tree="tree"),
        # prompts of several sequences
        rope("rope-prompts-8x2048", 8, 2048, 0, 8, 1, 256, 64),
        # three continuations of one prefix
        pages("pages-1x3", 1, 3, 816, 48, 7, 33, 18, 1, 256, 64),
        # eight robots' prefixes, one continuation each, a draft of 17 of which most is kept
        pages("pages-8x1", 8, 1, 816, 17, 9, 17, 18, 1, 256, 16),
        # half of the tokens behind the first camera view dropped for thirty-two continuations
        pages("pages-16x2", 16, 2, 816, 560, 5, 64, 18, 1, 256, 64),
    ]


HEADS = [(8, 1, 256), (16, 4, 128), (32, 8, 128), (14, 2, 64), (8, 8, 128), (12, 12, 64), (16, 2, 256)]


def spread(rng, lo, hi):
    """A whole number of lo .. hi, even over the logarithm."""
    return min(hi, int(lo * ((hi + 1) / lo) ** rng.random()))


def draw(rng):
    op = rng.choices(["attend", "rope", "pages"], weights=[5, 3, 2])[0]
    page, dtype = rng.choice([16, 32, 64, 128]), rng.choice(["bf16", "bf16", "f16"])
    if op == "pages":
        seqs, forks, longest = spread(rng, 1, 12), rng.randint(1, 3), spread(rng, 40, 816)
        c = pages("", seqs, forks, longest, spread(rng, 1, longest), rng.randint(1, 9), rng.randint(0, 64), rng.randint(1, 18),
                  *rng.choice([(1, 256), (1, 256), (4, 64), (2, 128)]), page, dtype)
    else:
        heads = rng.choice(HEADS[:1] + HEADS)
        per_token = heads[1] * heads[2]
        if op == "attend":
            seqs = spread(rng, 1, 64)
            longest = spread(rng, 1, max(1, min(16384, 64 * 8192 * 256 // (seqs * per_token))))
            nodes = spread(rng, 1, max(1, min(200, 8 * 64 * 16384 * 2048 // (seqs * longest * heads[0] * heads[2]))))
            c = attend("", seqs, nodes, longest, *heads, page, dtype, rng.random() < 0.7, rng.choice(["chain", "tree", "tree", "holes"]))
        else:
            seqs = spread(rng, 1, 64)
            nodes = spread(rng, 1, max(1, min(2048, 8 * 2048 * 2560 // (seqs * (heads[0] + 2 * heads[1]) * heads[2]))))
            longest = rng.choice([0, spread(rng, 1, 4096)])
            c = rope("", seqs, nodes, longest, *heads, page, dtype, rng.random() < 0.7, heads[2] // rng.choice([1, 1, 2]),
                     rng.random() < 0.4, rng.choice(["chain", "tree"]))
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------- what a case's sizes are
def ragged(n, most, on):
    """n numbers of 1 .. most, the first of them most; spread evenly and in no order."""
    return [most if not on or i == 0 or most == 0 else 1 + int((most - 1) * (i * 0.6180339887 % 1.0)) for i in range(n)]


def lengths(case):
    out = ragged(case["seqs"], case["longest"], case.get("ragged", True))
    if case.get("tree") == "holes" and case["seqs"] > 1:
        out[-1] = 0
    return out


def rows(case):
    return ragged(case["seqs"], case["nodes"], case["ragged"])


def kept(case, length):
    """The tail of a sequence and which of its positions stay, counted from the tail's first."""
    tail = min(case["tail"], length)
    return tail, [i for i in range(tail) if i * 7 % 10 < case["tenths"]]


def ceil_div(a, b):
    return -(-a // b)


def work(case):
    e = 2
    if case["op"] == "pages":
        moved = 0
        for n in lengths(case):
            tail, keep = kept(case, n)
            moved += case["forks"] * sum(1 for i, k in enumerate(keep) if i != k)
        row = case["layers"] * case["kv_heads"] * case["head_dim"] * 2 * e
        return {"bytes": 2 * moved * row + 8 * sum(ceil_div(n, case["page"]) for n in lengths(case)) * (1 + case["forks"]), "flops": 0}
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    n = sum(rows(case))
    if case["op"] == "rope":
        return {"bytes": 2 * e * n * (h + 2 * hk) * d, "flops": 10 * n * (h + hk) * d}
    held = sum(a + b for a, b in zip(lengths(case), rows(case)))
    pairs = sum(a * b + b * (b + 1) / 2 if case["tree"] == "chain" else a * b + b for a, b in zip(lengths(case), rows(case)))
    return {"bytes": held * hk * d * 2 * e + 2 * n * h * d * e, "flops": int(4 * h * d * pairs)}


# ---------------------------------------------------------------------------------------- inputs
def make_cache(case, gen, layers, room, spare=0):
    """Pages in random order for sequences of room[i] positions, all of them holding values."""
    page, hk, d = case["page"], case["kv_heads"], case["head_dim"]
    need = [ceil_div(r, page) for r in room]
    n_pages = max(1, sum(need) + spare)
    dtype = DTYPES[case["dtype"]]
    k, v = (torch.empty((layers, n_pages, page, hk, d), dtype=dtype, device="cuda") for _ in range(2))
    for t in (k, v):
        for layer in t:
            layer.copy_(torch.randn(layer.shape, generator=gen, device="cuda"))
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(room), max(1, max(need))), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs[order[:at].long()] = 1
    return k, v, table, refs


def make_tree(case, gen, count):
    """Who sees whom among `count` drafted tokens [count, count], and their depths."""
    if case["tree"] == "chain":
        return torch.ones((count, count), dtype=torch.bool, device="cuda").tril(), torch.arange(count, device="cuda")
    parents = (torch.rand(count, generator=gen, device="cuda") * torch.arange(count, device="cuda")).long().tolist()
    sees, depth = torch.zeros((count, count), dtype=torch.bool), [0] * count
    for i in range(count):
        if i:
            sees[i] = sees[parents[i]]
            depth[i] = depth[parents[i]] + 1
        sees[i, i] = True
    if case["tree"] == "holes":
        sees[::5] = False
    return sees.cuda(), torch.tensor(depth, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    lens, page, hk, d, dtype = lengths(case), case["page"], case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]]
    st = {"case": case, "lens": lens}

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    if case["op"] == "pages":
        seqs, forks = case["seqs"], case["forks"]
        tails = [kept(case, n) for n in lens for _ in range(forks)]
        most = max(ceil_div(n + case["extra"], page) for n in lens)
        k, v, table, refs = make_cache(case, gen, case["layers"], lens, spare=seqs * forks * (most + 1) + 2)
        wide = torch.full((seqs * (1 + forks), most + 1), -1, dtype=torch.int32, device="cuda")
        wide[:seqs, :table.shape[1]] = table
        src = [i for i in range(seqs) for _ in range(forks)]
        all_seqs = seqs * (1 + forks)
        start, n_keep, extra = [0] * all_seqs, [-1] * all_seqs, [-1] * all_seqs
        keep = torch.zeros((all_seqs, max(1, max(len(t[1]) for t in tails))), dtype=torch.int32)
        for j, (tail, stay) in enumerate(tails):
            start[seqs + j], n_keep[seqs + j], extra[seqs + j] = lens[src[j]] - tail, len(stay), case["extra"]
            keep[seqs + j, :len(stay)] = torch.tensor(stay, dtype=torch.int32)
        st |= {"k": k, "v": v, "table": wide, "refs": refs, "length": ints(lens + [0] * (seqs * forks)), "src": ints(src),
               "dst": ints(range(seqs, all_seqs)), "start": ints(start), "n_keep": ints(n_keep), "keep": keep.cuda(), "extra": ints(extra)}
    else:
        counts = rows(case)
        layers = 1
        k, v, table, refs = make_cache(case, gen, layers, [a + b for a, b in zip(lens, counts)], spare=2)
        n = sum(counts)
        starts = [0]
        for c in counts:
            starts.append(starts[-1] + c)
        st |= {"k": k, "v": v, "table": table, "refs": refs, "length": ints(lens), "counts": counts, "starts": starts,
               "row_start": ints(starts), "most": max(counts)}
        trees = [make_tree(case, gen, c) for c in counts]
        if case["op"] == "attend":
            st["sees"] = [t[0] for t in trees]
            st["mask"] = None
            if case["tree"] != "chain":
                words = ceil_div(max(counts), 32)
                bits = torch.zeros((n, words * 32), dtype=torch.int64, device="cuda")
                for i, t in enumerate(trees):
                    bits[starts[i]:starts[i + 1], :counts[i]] = t[0]
                m = (bits.view(n, words, 32) << torch.arange(32, device="cuda")).sum(-1)
                st["mask"] = torch.where(m >= 2 ** 31, m - 2 ** 32, m).to(torch.int32)
            st["q"] = (1.5 * torch.randn((n, case["heads"], d), generator=gen, device="cuda")).to(dtype)
            st["out"] = torch.empty_like(st["q"])
        else:
            h = case["heads"]
            # one row of the fused projection holds q, k and v of a token
            qkv = (2.0 * torch.randn((n, (h + 2 * hk) * d), generator=gen, device="cuda")).to(dtype)
            st["qkv"] = qkv
            st["q"], st["kk"], st["vv"] = (x.unflatten(1, (-1, d)) for x in qkv.split([h * d, hk * d, hk * d], 1))
            st["positions"] = None
            if case["tree"] != "chain":
                st["positions"] = torch.cat([lens[i] + t[1] for i, t in enumerate(trees)]).to(torch.int32)
            st["q_gain"], st["k_gain"] = (0.1 * torch.randn(d, generator=gen, device="cuda") for _ in range(2))
            st["out"] = torch.empty((n, h, d), dtype=dtype, device="cuda")
    if own:
        from paper_2510_26742_amd import binding
        st["pages"] = binding.Pages(st["k"], st["v"], st["table"], st["length"], st["refs"])
    return st


# ---------------------------------------------------------------------------------------- one pass
def run(st):
    if own:
        return run_own(st)
    return {"attend": plain_attend, "rope": plain_rope, "pages": plain_pages}[st["case"]["op"]](st)


def run_own(st):
    from paper_2510_26742_amd import binding
    case, p, stream = st["case"], st["pages"], torch.cuda.current_stream()
    if case["op"] == "attend":
        binding.pi0_tree_attention(p, 0, st["q"], st["row_start"], st["most"], mask=st["mask"], out=st["out"], stream=stream)
        return st["out"]
    if case["op"] == "rope":
        binding.pi0_qk_norm_rope(p, 0, st["q"], st["kk"], st["vv"], st["row_start"], st["most"], out=st["out"], positions=st["positions"],
                                 q_gain=st["q_gain"], k_gain=st["k_gain"], rope_dim=case["rope_dim"], interleaved=case["interleaved"],
                                 stream=stream)
        return {"q": st["out"], "k": st["k"], "v": st["v"]}
    p.pi0_pages_fork(st["src"], st["dst"], stream=stream)
    p.pi0_pages_compact(st["keep"], st["n_keep"], start=st["start"], stream=stream)
    p.pi0_pages_reserve(st["extra"], stream=stream)
    return cache_outputs(st)


def cache_outputs(st):
    return {"table": st["table"], "length": st["length"], "refs": st["refs"], "k": st["k"], "v": st["v"]}


def plain_attend(st):
    case = st["case"]
    hk, d, page = case["kv_heads"], case["head_dim"], case["page"]
    g = case["heads"] // hk
    for i, (length, n) in enumerate(zip(st["lens"], st["counts"])):
        total = length + n
        held = st["table"][i, :ceil_div(total, page)].long()
        k, v = (t[0][held].flatten(0, 1)[:total].float().transpose(0, 1) for t in (st["k"], st["v"]))
        q = st["q"][st["starts"][i]:st["starts"][i + 1]].float().view(n, hk, g, d).permute(1, 0, 2, 3).reshape(hk, n * g, d)
        s = torch.matmul(q, k.transpose(1, 2).contiguous()) * d ** -0.5
        seen = torch.cat([torch.ones((n, length), dtype=torch.bool, device="cuda"), st["sees"][i]], 1)
        seen = seen[:, None].expand(n, g, total).reshape(n * g, total)
        s = torch.where(seen, s, float("-inf"))
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - torch.where(top == float("-inf"), 0.0, top))
        total_p = p.sum(-1, keepdim=True)
        o = torch.matmul(p, v.contiguous()) / torch.where(total_p == 0, 1.0, total_p)
        st["out"][st["starts"][i]:st["starts"][i + 1]] = o.view(hk, n, g, d).permute(1, 0, 2, 3).reshape(n, hk * g, d).to(st["out"].dtype)
    return st["out"]


def token_places(st, i):
    """Pages and rows inside them of a sequence's new tokens."""
    at = st["lens"][i] + torch.arange(st["counts"][i], device="cuda")
    page = st["case"]["page"]
    return st["table"][i].long()[at // page], at % page


def plain_positions(st):
    if st["positions"] is not None:
        return st["positions"]
    return torch.cat([length + torch.arange(n, device="cuda") for length, n in zip(st["lens"], st["counts"])])


def plain_rope(st):
    case = st["case"]
    r = case["rope_dim"]
    angle = plain_positions(st).double()[:, None] * 10000.0 ** (-torch.arange(0, r, 2, device="cuda").double() / r)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def rotated(x, gain):
        x = x.float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * (1.0 + gain)
        a, b = (x[..., :r:2], x[..., 1:r:2]) if case["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
        a, b = a * cos - b * sin, a * sin + b * cos
        turned = torch.stack([a, b], -1).flatten(-2) if case["interleaved"] else torch.cat([a, b], -1)
        return torch.cat([turned, x[..., r:]], -1).to(st["out"].dtype)

    st["out"].copy_(rotated(st["q"], st["q_gain"]))
    k = rotated(st["kk"], st["k_gain"])
    for i in range(len(st["lens"])):
        where, rows_of = token_places(st, i), slice(st["starts"][i], st["starts"][i + 1])
        st["k"][0][where] = k[rows_of]
        st["v"][0][where] = st["vv"][rows_of]
    return {"q": st["out"], "k": st["k"], "v": st["v"]}


def plain_pages(st):
    """Page tables are kept on the host by a program without the operators: read, planned, written back, rows moved."""
    case = st["case"]
    page = case["page"]
    table, length, refs = st["table"].tolist(), st["length"].tolist(), st["refs"].tolist()
    held = [[p for p in row if p >= 0] for row in table]
    for s, d in zip(st["src"].tolist(), st["dst"].tolist()):
        for p in held[d]:
            refs[p] -= 1
        held[d] = held[s][:ceil_div(length[s], page)]
        for p in held[d]:
            refs[p] += 1
        length[d] = length[s]

    def copy_rows(sources, targets):
        if sources:
            a, b = (torch.tensor(x, device="cuda").unbind(1) for x in (sources, targets))
            for t in (st["k"], st["v"]):
                for layer in t:
                    layer[b[0], b[1]] = layer[a[0], a[1]]

    def fresh(count):
        free = [p for p, n in enumerate(refs) if n == 0]
        assert len(free) >= count, "no pages left"
        return iter(free)

    # compaction: the tail's kept positions close up; shared pages whose rows change are replaced
    sources, targets, gone, starts = [], [], [], st["start"].tolist()
    plans = []
    for s, (n, keep) in enumerate(zip(st["n_keep"].tolist(), st["keep"].tolist())):
        if n < 0:
            continue
        first = next((i for i in range(n) if keep[i] != i), n)
        begin, end = starts[s] + first, starts[s] + n
        new = [i for i in range(begin // page, ceil_div(end, page)) if begin < end and refs[held[s][i]] > 1]
        plans.append((s, keep, begin, end, new))
    free = fresh(sum(len(p[4]) for p in plans))
    for s, keep, begin, end, new in plans:
        old, mine = held[s], list(held[s])
        for i in new:
            mine[i] = next(free)
            gone.append(old[i])
        for pos in range(begin // page * page if begin // page in new else begin, end):
            src = pos if pos < begin else starts[s] + keep[pos - starts[s]]
            sources.append((old[src // page], src % page))
            targets.append((mine[pos // page], pos % page))
        gone += mine[ceil_div(end, page):]
        held[s], length[s] = mine[:ceil_div(end, page)], end
        for i in new:
            refs[mine[i]] = 1
    copy_rows(sources, targets)
    for p in gone:
        refs[p] -= 1

    # room for the next tokens: new pages, and own copies of shared pages that they will be written to
    plans, sources, targets, gone = [], [], [], []
    for s, extra in enumerate(st["extra"].tolist()):
        if extra < 0:
            continue
        want = ceil_div(length[s] + extra, page)
        shared = [i for i in range(length[s] // page, min(want, len(held[s]))) if extra > 0 and refs[held[s][i]] > 1]
        plans.append((s, shared, max(0, want - len(held[s]))))
    free = fresh(sum(len(p[1]) + p[2] for p in plans))
    for s, shared, more in plans:
        for i in shared:
            q = next(free)
            for r in range(min(page, length[s] - i * page)):
                sources.append((held[s][i], r))
                targets.append((q, r))
            gone.append(held[s][i])
            held[s][i] = q
            refs[q] = 1
        for _ in range(more):
            held[s].append(next(free))
            refs[held[s][-1]] = 1
    copy_rows(sources, targets)
    for p in gone:
        refs[p] -= 1
    wide = len(table[0])
    st["table"].copy_(torch.tensor([row + [-1] * (wide - len(row)) for row in held], dtype=torch.int32))
    st["length"].copy_(torch.tensor(length, dtype=torch.int32))
    st["refs"].copy_(torch.tensor(refs, dtype=torch.int32))
    return cache_outputs(st)


# ---------------------------------------------------------------------------------------- the definition, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"attend": exact_attend, "rope": exact_rope, "pages": exact_pages}[case["op"]](st)


def flat_rows(st, i, count):
    """Rows of the flattened pool [n_pages * page] that hold a sequence's first `count` positions."""
    page, table = st["case"]["page"], st["table"][i].tolist()
    return torch.tensor([table[p // page] * page + p % page for p in range(count)], dtype=torch.long, device="cuda")


def exact_attend(st):
    case = st["case"]
    per = case["heads"] // case["kv_heads"]
    d = case["head_dim"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for i, (length, n) in enumerate(zip(st["lens"], st["counts"])):
        at = flat_rows(st, i, length + n)
        open_ = torch.ones((n, length + n), dtype=torch.float64, device="cuda")
        open_[:, length:] = st["sees"][i].double()
        for h in range(case["heads"]):
            keys, values = (t[0, :, :, h // per].reshape(-1, d)[at].double() for t in (st["k"], st["v"]))
            logits = st["q"][st["starts"][i]:st["starts"][i + 1], h].double() @ keys.t().contiguous() / d ** 0.5
            weight = torch.exp(logits - logits.max()) * open_      # far from underflow: logits of order ten
            whole = weight.sum(1)
            some = whole > 0
            out[st["starts"][i]:st["starts"][i + 1], h][some] = (weight @ values)[some] / whole[some][:, None]
    return out


def exact_rope(st):
    case = st["case"]
    r = case["rope_dim"]
    q, k, v = (t.double() for t in (st["q"], st["k"], st["v"]))
    where = torch.cat([flat_rows(st, i, a + b)[a:] for i, (a, b) in enumerate(zip(st["lens"], st["counts"]))])
    position = plain_positions(st).double()
    turn = torch.stack([torch.polar(torch.ones_like(position), position * 10000.0 ** (-2.0 * i / r)) for i in range(r // 2)], 1)[:, None]

    def normed(x, gain):
        x = x.double()
        return x / (x.square().sum(-1, keepdim=True) / x.shape[-1] + 1e-6).sqrt() * (1.0 + gain.double())

    def turned(x):
        x = x.clone()
        first = slice(0, r, 2) if case["interleaved"] else slice(0, r // 2)
        second = slice(1, r, 2) if case["interleaved"] else slice(r // 2, r)
        z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    k[0].view(-1, *k.shape[3:])[where] = turned(normed(st["kk"], st["k_gain"]))
    v[0].view(-1, *v.shape[3:])[where] = st["vv"].double()
    return {"q": turned(normed(q, st["q_gain"])), "k": k, "v": v}


def exact_pages(st):
    """Nothing is computed: whole numbers follow from the plan, values are copies of values."""
    return None
