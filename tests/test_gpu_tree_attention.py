"""GPU: attention of drafted tokens over pages against the definition in float64.

Bar.  With u = eps / 2 of the type: the weights of the second product are rounded, and their sum is that of the rounded ones, so
the result moves by at most u max|v - o| <= 2 u V, V the largest |v| that is seen; rounding it u |o| <= u V.  In fp32: a score is a sum
of d products, off by at most (d + 2) 2^-24 scale |q| |k|, which moves its weight by as much relatively and the result by twice that times V; the
running sums (n terms, rescaled now and then) n 2^-24 twice.  Sums of fp16 results near zero: half a step of the smallest number."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2510_26742_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def f64(t):
    return t.double().cpu().numpy()


def words(sees, most):
    """bool [n, n] -> int32 [n, words]"""
    n = sees.shape[0]
    out = np.zeros((n, -(-most // 32)), dtype=np.uint32)
    for i, j in zip(*np.nonzero(sees)):
        out[i, j // 32] |= np.uint32(1) << np.uint32(j % 32)
    return out.view(np.int32)


def tree(kind, n, rng):
    if kind == "chain":
        return np.tril(np.ones((n, n), dtype=bool))
    sees = np.zeros((n, n), dtype=bool)
    for i in range(n):
        if i:
            sees[i] = sees[int(rng.integers(i))]
        sees[i, i] = True
    if kind == "holes":
        sees[::3] = False
    if kind == "random":
        sees = rng.random((n, n)) < 0.3
    return sees


class Case:
    """A cache whose unseen rows are NaN, rows of queries with rows around them that belong to nobody."""

    def __init__(self, seed, lengths, counts, heads, kv_heads, d, page, dtype, kind="tree", layers=1, scatter=(0, 1, 2, 3), spread=1.0, max_rows=None):
        rng = self.rng = np.random.default_rng(seed)
        self.lengths, self.counts, self.page, self.d, self.dtype, self.kind = lengths, counts, page, d, TYPES[dtype], kind
        need = [-(-(a + b) // page) for a, b in zip(lengths, counts)]
        n_pages = sum(need) + 1
        self.table = np.full((len(lengths), max(max(need), 1) + 2), -1)
        order, at = rng.permutation(n_pages), 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        shape = (layers, n_pages, page, kv_heads)
        pools = [torch.empty([shape[i] for i in scatter] + [d], dtype=self.dtype, device=DEV).permute(*[scatter.index(i) for i in range(4)], 4) for _ in range(2)]
        self.layer = layers - 1
        for t in pools:
            t.fill_(float("nan"))
        self.k, self.v = [], []
        for s, (a, b) in enumerate(zip(lengths, counts)):
            pos = np.arange(a + b)
            where = torch.from_numpy(self.table[s][pos // page]).to(DEV), torch.from_numpy(pos % page).to(DEV)
            for t, mine in zip(pools, (self.k, self.v)):
                x = torch.from_numpy(rng.standard_normal((a + b, kv_heads, d))).to(DEV, self.dtype)
                t[self.layer][where] = x
                mine.append(f64(x))
        self.pages = binding.Pages(*pools, ints(self.table), ints(lengths), ints(np.ones(n_pages)))
        self.before, n = 3, sum(counts) + 5
        self.starts = self.before + np.concatenate([[0], np.cumsum(counts)])
        self.most = max(counts) if max_rows is None else max_rows
        self.q = torch.from_numpy(rng.standard_normal((n, heads, d)) * spread).to(DEV, self.dtype)
        self.sees = [tree(kind, c, rng) for c in counts]
        self.mask = None
        if kind != "chain":
            m = np.full((n, -(-max(self.most, 1) // 32)), -1, dtype=np.int32)
            for s, c in enumerate(counts):
                m[self.starts[s]:self.starts[s + 1]] = words(self.sees[s], self.most)[:, :m.shape[1]]
            self.mask = ints(m)
        self.out = torch.full((n, heads, d), 7.0, dtype=self.dtype, device=DEV)

    def run(self, **kw):
        return binding.pi0_tree_attention(self.pages, self.layer, self.q, ints(self.starts), self.most, mask=self.mask, out=self.out, **kw)

    def seen(self, s):
        a, b = self.lengths[s], self.counts[s]
        return np.concatenate([np.ones((b, a), dtype=bool), self.sees[s]], 1)

    def check(self, scale=None, seen=None):
        scale = self.d ** -0.5 if scale is None else scale
        got = f64(self.out)
        assert (got[:self.before] == 7).all() and (got[self.starts[-1]:] == 7).all()
        u, worst = torch.finfo(self.dtype).eps / 2, 0.0
        for s, c in enumerate(self.counts):
            if c == 0:
                continue
            see = self.seen(s) if seen is None else seen(s)
            q = f64(self.q[self.starts[s]:self.starts[s + 1]])
            want = paged.attention(q, self.k[s], self.v[s], see, scale)
            any_seen = see.any(0)
            if not any_seen.any():
                assert (got[self.starts[s]:self.starts[s + 1]] == 0).all()
                continue
            big = np.abs(self.v[s][any_seen]).max()
            score = abs(scale) * np.sqrt((q ** 2).sum(-1).max() * (self.k[s][any_seen] ** 2).sum(-1).max())
            n = see.shape[1]
            bar = (3 * u + 2.0 ** -24 * (2 * (self.d + 2) * score + 2 * n)) * big + (2.0 ** -25 if u < 2.0 ** -9 else 0.0)
            delta = np.abs(got[self.starts[s]:self.starts[s + 1]] - want)
            worst = max(worst, delta.max() / bar)
            assert (got[self.starts[s]:self.starts[s + 1]][~see.any(1)] == 0).all()
        print(f"[attention] worst {worst:.3f} of the bar", flush=True)
        assert worst <= 1.0


CASES = [  # lengths, counts, heads, kv heads, head dim, page, type, mask
    dict(lengths=[816], counts=[1], heads=8, kv_heads=1, d=256, page=64, dtype="bf16", kind="chain"),
    dict(lengths=[0], counts=[1], heads=8, kv_heads=1, d=256, page=64, dtype="bf16", kind="chain"),
    dict(lengths=[0, 1, 31, 32, 33, 63, 64, 65, 0], counts=[1, 1, 1, 0, 2, 1, 1, 1, 3], heads=8, kv_heads=1, d=256, page=16, dtype="bf16"),
    dict(lengths=[0, 5, 200], counts=[7, 4, 6], heads=4, kv_heads=4, d=64, page=16, dtype="f16", kind="holes"),
    dict(lengths=[700], counts=[64], heads=8, kv_heads=1, d=256, page=32, dtype="bf16"),
    dict(lengths=[100, 513], counts=[5, 33], heads=14, kv_heads=2, d=64, page=128, dtype="bf16", kind="random"),
    dict(lengths=[257, 0, 1000], counts=[33, 17, 1], heads=16, kv_heads=4, d=128, page=16, dtype="f16", kind="holes"),
    dict(lengths=[40], counts=[200], heads=4, kv_heads=2, d=128, page=64, dtype="bf16", kind="tree"),
    dict(lengths=[3, 90], counts=[130, 77], heads=3, kv_heads=3, d=256, page=256, dtype="f16", kind="chain"),
    dict(lengths=[5000, 3, 1777], counts=[2, 2, 2], heads=8, kv_heads=1, d=256, page=64, dtype="bf16"),
    dict(lengths=[12000], counts=[9], heads=32, kv_heads=8, d=128, page=32, dtype="bf16"),
    dict(lengths=[60] * 50, counts=[1, 2, 0, 3, 1] * 10, heads=12, kv_heads=12, d=64, page=16, dtype="bf16", kind="random"),
    dict(lengths=[30], counts=[1000], heads=2, kv_heads=1, d=64, page=64, dtype="f16", kind="chain"),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_against_the_definition(i):
    print("[gpu] tree_attention", CASES[i], flush=True)
    c = Case(i, **CASES[i])
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 256), ("f16", 128), ("bf16", 64)])
@pytest.mark.parametrize("rows", [15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 257])
@pytest.mark.parametrize("seqs", [1, 4])
def test_any_number_of_rows(dtype, d, rows, seqs):
    """One head per token, so that every number of rows in a tile, and of tiles, occurs; one sequence, and four with fewer and fewer."""
    print("[gpu] tree_attention", dtype, d, rows, seqs, flush=True)
    counts = [rows, 1, rows // 2, rows - 1][:seqs]
    c = Case(rows, [900, 33, 0, 350][:seqs], counts, 1, 1, d, 16, dtype, kind="random")
    c.run()
    c.check()


@pytest.mark.parametrize("n_seqs", [64, 65, 300, 1024])
def test_many_sequences(n_seqs):
    rng = np.random.default_rng(n_seqs)
    lengths, counts = rng.integers(0, 90, n_seqs).tolist(), rng.integers(0, 3, n_seqs).tolist()
    lengths[0], lengths[-1], counts[-1] = 2000, 700, 2
    c = Case(n_seqs, lengths, counts, 4, 2, 64, 32, "f16", kind="tree")
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("seqs,count", [(1, 3), (4, 20)])
def test_scores_that_grow_along_the_keys(dtype, seqs, count):
    """Later keys outweigh all in front of them time and again: what has been summed is scaled down over and over."""
    c = Case(70, [1500, 700, 64, 3][:seqs], [count] * seqs, 8, 1, 256, 64, dtype, kind="chain")
    for s in range(seqs):
        n = c.lengths[s] + count
        pos = np.arange(n)
        where = torch.from_numpy(c.table[s][pos // 64]).to(DEV), torch.from_numpy(pos % 64).to(DEV)
        k = torch.from_numpy(c.k[s]).to(DEV) + 0.02 * torch.arange(n, device=DEV)[:, None, None]
        c.pages.k[0][where] = k.to(c.dtype)
        c.k[s] = f64(c.pages.k[0][where])
    c.q.abs_()
    c.run()
    c.check()


@pytest.mark.parametrize("spread,scale", [(30.0, None), (1.0, -0.2), (1.0, 0.0), (0.0, None)])
def test_sharp_negative_and_flat(spread, scale):
    c = Case(50, [300, 70], [5, 40], 8, 1, 256, 32, "bf16", spread=spread)
    c.run(scale=scale)
    c.check(scale=scale)


@pytest.mark.parametrize("scatter", [(0, 1, 3, 2), (1, 0, 2, 3), (3, 0, 1, 2)])
def test_layouts_layers_and_slices(scatter):
    """Heads outside tokens, layers inside pages, heads outermost; queries as a slice of a fused row, results into one."""
    c = Case(60, [100, 30], [3, 35], 6, 2, 128, 16, "bf16", layers=3, scatter=scatter)
    wide = torch.zeros((c.q.shape[0], 10, 128), dtype=c.dtype, device=DEV)
    wide[:, 2:8] = c.q
    binding.pi0_tree_attention(c.pages, 2, wide[:, 2:8], ints(c.starts), c.most, mask=c.mask, out=wide[:, 2:8])       # and in place
    c.out[c.starts[0]:c.starts[-1]] = wide[c.starts[0]:c.starts[-1], 2:8]
    c.check()
    assert not wide[:, :2].any() and not wide[:, 8:].any()


@pytest.mark.parametrize("dtype,d", [("bf16", 256), ("f16", 128), ("bf16", 64)])
def test_what_is_not_seen_may_be_anything(dtype, d):
    """NaN and infinities in keys and values of drafts, next to rows that see them and rows that do not."""
    c = Case(70, [37, 3], [40, 6], 8, 2, d, 16, dtype, kind="tree")
    for s, (a, b) in enumerate(zip(c.lengths, c.counts)):
        sick = {1: ("k", float("nan")), 3: ("v", float("nan")), 5: ("v", float("inf")), b - 1: ("v", float("-inf"))}
        for node, (pool, x) in sick.items():
            pos = a + node
            getattr(c.pages, pool)[0, int(c.table[s, pos // 16]), pos % 16, :, 3:7] = x
            (c.k if pool == "k" else c.v)[s][pos, :, 3:7] = x
    c.run()
    got = f64(c.out)
    for s, (a, b) in enumerate(zip(c.lengths, c.counts)):
        sees = c.sees[s]
        poisoned = sees[:, [1, 3, 5, b - 1]].any(1)
        mine = got[c.starts[s]:c.starts[s + 1]]
        assert poisoned.any() and not poisoned.all()
        with np.errstate(invalid="ignore"):
            want = paged.attention(f64(c.q[c.starts[s]:c.starts[s + 1]]), c.k[s], c.v[s], c.seen(s), c.d ** -0.5)
        assert np.array_equal(np.isnan(mine), np.isnan(want)) and np.array_equal(np.isinf(mine), np.isinf(want))
        assert np.isfinite(mine[~poisoned]).all()
        fine = np.isfinite(want)
        assert np.abs(mine[fine] - want[fine]).max() <= 2.0 ** -7 * 6


def test_committed_values_that_are_no_numbers_reach_every_row():
    for at in (3, 36):                        # in a tile of its own, and in one that drafts begin in
        c = Case(75, [37], [6], 8, 2, 128, 16, "bf16")
        c.pages.v[0, int(c.table[0, at // 16]), at % 16, 1, 5] = float("-inf")
        c.run()
        got = f64(c.out)[c.starts[0]:c.starts[1]]
        assert np.isneginf(got[:, 4:, 5]).all()
        got[:, 4:, 5] = 0
        assert np.isfinite(got).all()


def test_positions_without_a_page_are_not_seen():
    c = Case(80, [100, 64], [4, 4], 8, 1, 256, 16, "bf16")
    c.pages.table[0, 2] = -1
    c.pages.table[0, 5] = 1 << 30
    c.pages.table[1, 0] = c.pages.k.shape[1]       # one behind the last
    gone = [[*range(32, 48), *range(80, 96)], [*range(16)]]

    def seen(s):
        x = c.seen(s).copy()
        x[:, gone[s]] = False
        return x
    c.run()
    c.check(seen=seen)


def test_more_tokens_than_max_rows_and_starts_that_make_no_sense():
    """Tokens behind max_rows are no rows and no keys; sequences outside the rows are none."""
    c = Case(90, [20, 20, 9, 30], [10, 50, 3, 4], 8, 1, 256, 16, "bf16", kind="chain", max_rows=12)
    whole = f64(c.out)
    c.run()
    got = f64(c.out)
    assert np.array_equal(got[c.starts[1] + 12:c.starts[2]], whole[c.starts[1] + 12:c.starts[2]])
    see = np.concatenate([np.ones((12, 20), dtype=bool), np.tril(np.ones((12, 12), dtype=bool))], 1)
    want = paged.attention(f64(c.q[c.starts[1]:c.starts[1] + 12]), c.k[1][:32], c.v[1][:32], see, 1 / 16)
    assert np.abs(got[c.starts[1]:c.starts[1] + 12] - want).max() <= 2.0 ** -7 * np.abs(c.v[1]).max()
    c.out.fill_(7.0)
    n = c.q.shape[0]
    binding.pi0_tree_attention(c.pages, 0, c.q, ints([-3, 2, 1, n + 9, n + 10]), 12, out=c.out)
    got = f64(c.out)
    rows = [bool((got[i] != 7).any()) for i in range(n)]
    assert rows == [1 <= i < 13 for i in range(n)]         # the third sequence's first twelve rows
    # that sequence holds 9 + 3 positions and NaN behind them: rows 1 .. 3 see the former only, the other nine also the latter
    assert np.isfinite(got[1:4]).all() and np.isnan(got[4:13]).all()


def test_pool_beyond_32_bits():
    """Pages whose offsets pass 2^32 bytes, in a pool of 2 x 5 GB."""
    d, page, n_pages = 256, 256, 40000
    k, v = (torch.zeros((1, n_pages, page, 1, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    rng = np.random.default_rng(11)
    table = np.array([[n_pages - 1, 3, 33000, -1]])
    pages = binding.Pages(k, v, ints(table), ints([600]), ints(np.ones(n_pages)))
    rows = [torch.from_numpy(rng.standard_normal((602, 1, d))).to(DEV, torch.bfloat16) for _ in range(2)]
    starts = ints([0, 2])
    q = torch.from_numpy(rng.standard_normal((2, 8, d))).to(DEV, torch.bfloat16)
    pos = np.arange(602)
    where = torch.from_numpy(table[0][pos // page]).to(DEV), torch.from_numpy(pos % page).to(DEV)
    k[0][where], v[0][where] = rows
    out = binding.pi0_tree_attention(pages, 0, q, starts, 2)
    see = np.concatenate([np.ones((2, 600), dtype=bool), np.tril(np.ones((2, 2), dtype=bool))], 1)
    want = paged.attention(f64(q), *[f64(t) for t in rows], see, 1 / 16)
    assert np.abs(f64(out) - want).max() <= 2.0 ** -7 * 6
    # keys and values that are appended there
    binding.pi0_qk_norm_rope(pages, 0, q, rows[0][:2], rows[1][:2], starts, 2, rope_dim=0)
    assert torch.equal(v[0, 33000, 600 - 512:602 - 512], rows[1][:2]) and torch.equal(k[0, 33000, 600 - 512:602 - 512], rows[0][:2])
    pages.pi0_pages_compact(ints([[1]]), ints([1]))
    pages.pi0_pages_status()
    assert torch.equal(v[0, 33000, 600 - 512], rows[1][1])


@pytest.mark.parametrize("d", [64, 128, 256])
def test_rows_as_far_apart_as_is_taken(d):
    """16 rows of a page 2^27 - 8 elements apart: the last offset inside a granule just fits 32 bits."""
    apart, rng = (1 << 27) - 8, np.random.default_rng(d)
    pools = [torch.empty(2 * 16 * apart, dtype=torch.bfloat16, device=DEV).as_strided((1, 2, 16, 1, d), (32 * apart, 16 * apart, apart, d, 1)) for _ in range(2)]
    held = [torch.from_numpy(rng.standard_normal((32, 1, d))).to(DEV, torch.bfloat16) for _ in range(2)]
    for t, x in zip(pools, held):
        t[0, 1], t[0, 0] = x[:16], x[16:]                       # the list is pages 1, 0
    pages = binding.Pages(*pools, ints([[1, 0]]), ints([29]), ints([1, 1]))
    q = torch.from_numpy(rng.standard_normal((3, 2, d))).to(DEV, torch.bfloat16)
    got = f64(binding.pi0_tree_attention(pages, 0, q, ints([0, 3]), 3))
    see = np.concatenate([np.ones((3, 29), dtype=bool), np.tril(np.ones((3, 3), dtype=bool))], 1)
    k, v = (f64(x) for x in held)
    want = paged.attention(f64(q), k, v, see, d ** -0.5)
    score = d ** -0.5 * np.sqrt((f64(q) ** 2).sum(-1).max() * (k ** 2).sum(-1).max())
    bar = (3 * 2.0 ** -8 + 2.0 ** -24 * (2 * (d + 2) * score + 64)) * np.abs(v).max()
    assert np.abs(got - want).max() <= bar


@pytest.mark.parametrize("seqs,count,heads,kv_heads,d", [(1, 70, 4, 1, 256), (4, 70, 4, 1, 128), (6, 33, 16, 4, 64)])
def test_results_in_the_place_of_the_queries(seqs, count, heads, kv_heads, d):
    """Several tiles of rows per sequence, units that one block has all of and units that many have a part in: the same bits."""
    c = Case(80, [2500, 10, 300, 64, 0, 31][:seqs], [count - 5 * s for s in range(seqs)], heads, kv_heads, d, 32, "bf16")
    c.run()
    c.check()
    q = c.q.clone()
    binding.pi0_tree_attention(c.pages, c.layer, q, ints(c.starts), c.most, mask=c.mask, out=q)
    mine = slice(int(c.starts[0]), int(c.starts[-1]))
    assert torch.equal(q[mine], c.out[mine]) and torch.equal(q[:c.before], c.q[:c.before]) and torch.equal(q[mine.stop:], c.q[mine.stop:])


def test_streams_and_replays():
    """Calls on two streams at once, and a graph replayed with other lengths, masks and pages, against eager calls bit for bit."""
    a, b = Case(101, [900, 40], [3, 9], 8, 1, 256, 32, "bf16"), Case(102, [50, 1200, 7], [20, 1, 2], 16, 4, 128, 16, "f16")
    for c in (a, b):
        c.run()
        c.want = c.out.clone()
    side = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip((a, b), side):
            c.out.fill_(7.0)
        torch.cuda.synchronize()
        for c, s in zip((a, b), side):
            with torch.cuda.stream(s):
                c.run(stream=s)
        torch.cuda.synchronize()
        for c in (a, b):
            assert torch.equal(c.out.view(torch.int16), c.want.view(torch.int16))
    starts = ints(a.starts)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side[0]):
        binding.pi0_tree_attention(a.pages, 0, a.q, starts, a.most, mask=a.mask, out=a.out, stream=side[0])
    for step, lengths in enumerate(([900, 40], [0, 0], [333, 41], [899, 1])):
        a.pages.length.copy_(ints(lengths))
        torch.cuda.synchronize()
        a.out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = a.out.clone()
        eager = torch.full_like(a.out, 7.0)
        binding.pi0_tree_attention(a.pages, 0, a.q, starts, a.most, mask=a.mask, out=eager)
        assert torch.equal(replayed.view(torch.int16), eager.view(torch.int16)), step
    same = [binding.pi0_tree_attention(a.pages, 0, a.q, starts, a.most, mask=a.mask)[a.before:a.starts[-1]].clone() for _ in range(3)]
    assert torch.equal(same[0].view(torch.int16), same[1].view(torch.int16)) and torch.equal(same[0].view(torch.int16), same[2].view(torch.int16))


def test_binding_refuses():
    c = Case(110, [10], [3], 4, 2, 64, 16, "bf16")
    s = ints(c.starts)
    for bad in (dict(q=c.q.half()), dict(q=c.q[:, :3]), dict(q=c.q.cpu()), dict(most=0), dict(most=1025), dict(mask=c.mask[:2]), dict(mask=c.mask.long()),
                dict(s=s[:1]), dict(layer=1), dict(out=c.out[:2]), dict(out=c.out.float()), dict(scale=float("nan"))):
        a = dict(q=c.q, s=s, most=3, layer=0)
        kw = {**dict(mask=c.mask), **{n: x for n, x in bad.items() if n not in a}}
        a.update({n: x for n, x in bad.items() if n in a})
        with pytest.raises(binding.Pi0Error) as e:
            binding.pi0_tree_attention(c.pages, a["layer"], a["q"], a["s"], a["most"], **kw)
        assert e.value.code == binding.PI0_EINVAL, bad


@pytest.mark.parametrize("seqs,count,heads,kv_heads,d", [(1, 70, 4, 1, 256), (1, 33, 4, 1, 128), (4, 70, 4, 1, 256), (4, 70, 4, 1, 64)])
def test_lanes_without_a_row_have_no_say(seqs, count, heads, kv_heads, d):
    """The last tile has fewer rows than lanes.  What the first token asks for - scores that grow along the keys, time and again - is nothing
    to the rows of other waves: the same bits whether it does or not."""
    print("[gpu] tree_attention idle lanes", seqs, count, d, flush=True)
    c = Case(120 + d, [2500, 10, 300, 64][:seqs], [count - 5 * s for s in range(seqs)], heads, kv_heads, d, 32, "bf16", kind="chain")
    c.run()
    want = c.out.clone()
    for s in range(seqs):
        c.q[c.starts[s]] *= 40
    c.run()
    c.check()
    for s in range(seqs):
        rest = slice(int(c.starts[s]) + 32 // heads, int(c.starts[s + 1]))      # 32 rows: the first wave's
        assert torch.equal(c.out[rest].view(torch.int16), want[rest].view(torch.int16))


@pytest.mark.parametrize("d,dtype", [(256, "bf16"), (128, "f16"), (64, "bf16")])
def test_in_place_where_blocks_have_many_units(d, dtype):
    """Two tiles of rows for each of 600 short sequences, the second hardly filled, sharp scores: a block has several units, and the first tile's
    results take their queries' place while others are at the second.  The same bits as beside them, time after time."""
    print("[gpu] tree_attention in place, many units", d, dtype, flush=True)
    rng = np.random.default_rng(d)
    c = Case(130, rng.integers(0, 48, 600).tolist(), [17] * 600, 8, 1, d, 16, dtype, spread=30.0)
    c.run()
    mine, starts = slice(int(c.starts[0]), int(c.starts[-1])), ints(c.starts)
    for _ in range(4):
        q = c.q.clone()
        binding.pi0_tree_attention(c.pages, c.layer, q, starts, c.most, mask=c.mask, out=q)
        assert torch.equal(q[mine].view(torch.int16), c.out[mine].view(torch.int16))
        assert torch.equal(q[:c.before], c.q[:c.before]) and torch.equal(q[mine.stop:], c.q[mine.stop:])


def test_axes_of_one_with_any_stride():
    """One token whose queries lie in a row of odd width, over one head, in one layer, whose axes have strides that say nothing."""
    rng = np.random.default_rng(140)
    k, v = (torch.from_numpy(rng.standard_normal((1, 4, 16, 64, 1))).to(DEV, torch.bfloat16).transpose(3, 4) for _ in range(2))
    v = v.as_strided(v.shape, (7, 16 * 64, 64, 3, 1))
    pages = binding.Pages(k, v, ints([[2, 0, 3, -1]]), ints([40]), ints([1, 0, 1, 1]))
    q = torch.from_numpy(rng.standard_normal(8 * 64 + 3)).to(DEV, torch.bfloat16).as_strided((1, 8, 64), (515, 64, 1))
    out = binding.pi0_tree_attention(pages, 0, q, ints([0, 1]), 1)
    held = [f64(t[0, [2, 0, 3]].reshape(-1, 1, 64))[:41] for t in (k, v)]
    want = paged.attention(f64(q), *held, np.ones((1, 41), dtype=bool), 0.125)
    assert np.abs(f64(out) - want).max() <= 2.0 ** -7 * np.abs(held[1]).max()
    binding.pi0_qk_norm_rope(pages, 0, q, q[:, :1], q[:, 1:2], ints([0, 1]), 1, rope_dim=0)
    assert torch.equal(k[0, 3, 8, 0], q[0, 0]) and torch.equal(v[0, 3, 8, 0], q[0, 1])


@pytest.mark.parametrize("d,dtype", [(256, "bf16"), (128, "f16"), (64, "bf16")])
def test_missing_pages_where_rows_are_many(d, dtype):
    """Tiles of 128 rows, whose scores run a granule ahead: halves of a unit's first, middle and last granules are on no page, whole granules, and
    a sequence's every page."""
    c = Case(150, [100, 64, 0, 333, 40], [20, 20, 33, 17, 20], 8, 1, d, 16, dtype, kind="random")
    gone = [[0, 5, 7], [0, 1, 4], [0, 2], [1, 2, 3, 10, 21], [0, 1, 2, 3]]
    for s, idx in enumerate(gone):
        for i in idx:
            c.pages.table[s, i] = [-1, c.pages.k.shape[1], 1 << 30][i % 3]

    def seen(s):
        x = c.seen(s).copy()
        for i in gone[s]:
            x[:, 16 * i:16 * i + 16] = False
        return x
    c.run()
    c.check(seen=seen)


def test_as_many_rows_as_there_can_be():
    """1024 tokens of 1024 heads over one: 2^20 rows.  Queries of zero make a token's result the mean of the values that it sees, here half its number -
    a different one for each token, and fp16 tells them apart."""
    n, d = 1024, 64
    k = torch.zeros((1, 65, 16, 1, d), dtype=torch.float16, device=DEV)
    v = torch.arange(65 * 16, device=DEV).reshape(1, 65, 16, 1, 1).expand(1, 65, 16, 1, d).to(torch.float16).contiguous()
    pages = binding.Pages(k, v, ints([np.arange(65)]), ints([0]), ints(np.ones(65)))
    q = torch.zeros((n, n, d), dtype=torch.float16, device=DEV)
    out = torch.full_like(q, float("nan"))
    binding.pi0_tree_attention(pages, 0, q, ints([0, n]), n, out=out)
    # sums of whole numbers, times a power of two, are exact in 32 bits; the quotient is off by 2^-14 at most, and halves below 512 are numbers of fp16
    want = (torch.arange(n, device=DEV, dtype=torch.float32) / 2).to(torch.float16)
    assert torch.equal(out, want[:, None, None].expand(n, n, d))
