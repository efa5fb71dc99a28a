"""The operators of include/pi0_ops.h as far as they go without a GPU: what the library exports, what it refuses before
any GPU call, and the plain page bookkeeping that the GPU tests compare with."""
import copy
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from oracle import paged
from paper_2510_26742_amd import binding, synth

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000   # never dereferenced: every call below fails a check


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    return binding.lib()


def good(**kw):
    c = dict(d_k=FAKE, d_v=FAKE, d_table=FAKE, d_length=FAKE, d_refs=FAKE, d_status=FAKE, layer_stride=10 * 64 * 256, page_stride=64 * 256,
             token_stride=256, head_stride=256, dtype=0, layers=18, n_pages=10, page_tokens=64, kv_heads=1, head_dim=256, n_seqs=4, max_pages=5)
    return binding.PagesC(**{**c, **kw})


BAD_PAGES = [dict(d_k=None), dict(d_v=None), dict(d_table=None), dict(d_length=None), dict(d_refs=None), dict(d_status=None), dict(d_k=FAKE + 8),
             dict(d_v=FAKE + 2), dict(d_table=FAKE + 2), dict(dtype=2), dict(dtype=-1), dict(layers=0), dict(n_pages=0), dict(n_pages=(1 << 24) + 1),
             dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=512), dict(kv_heads=0), dict(kv_heads=257), dict(head_dim=72),
             dict(head_dim=96), dict(head_dim=512), dict(n_seqs=0), dict(n_seqs=1025), dict(max_pages=0), dict(max_pages=1 << 19),
             dict(token_stride=252), dict(token_stride=128), dict(page_stride=64 * 256 - 8), dict(page_stride=-64 * 256), dict(layer_stride=0),
             dict(kv_heads=2), dict(kv_heads=2, head_stride=0)]


def test_header_symbols_are_exported(L):
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "pi0_ops.h")).read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(pi0_[a-z_0-9]+)\s*\(", header)))
    assert declared == sorted(binding.OPS_EXPORTS)
    for name in declared:
        assert hasattr(L, name), name
    assert ctypes.sizeof(binding.PagesC) == 6 * 8 + 4 * 8 + 8 * 4 and ctypes.sizeof(binding.RowsC) == 32


def test_a_cache_that_is_none(L):
    ws = 1 << 30
    for kw in BAD_PAGES:
        p = ctypes.byref(good(**kw))
        assert L.pi0_pages_workspace_bytes(p) == 0, kw
        assert L.pi0_pages_reserve(p, FAKE, FAKE, ws, None) == binding.PI0_EINVAL, kw
        assert L.pi0_pages_fork(p, FAKE, FAKE, 1, None) == binding.PI0_EINVAL, kw
        assert L.pi0_pages_compact(p, None, FAKE, 1, FAKE, FAKE, ws, None) == binding.PI0_EINVAL, kw
        assert L.pi0_pages_status(p, None) == binding.PI0_EINVAL, kw
        assert L.pi0_tree_attention_workspace_bytes(p, 8, 1, 1) == 0, kw
    assert L.pi0_pages_workspace_bytes(None) == 0
    assert L.pi0_pages_status(None, None) == binding.PI0_EINVAL


@pytest.mark.parametrize("kw", [dict(), dict(kv_heads=4, head_dim=64, token_stride=256, head_stride=64),
                                dict(kv_heads=4, head_dim=64, token_stride=64, head_stride=64 * 64),               # heads outside tokens
                                dict(layer_stride=256, token_stride=18 * 256, page_stride=64 * 18 * 256),          # layers inside tokens
                                dict(layers=1, layer_stride=0), dict(n_pages=1, page_stride=0, layer_stride=64 * 256)])
def test_layouts_that_are_taken(L, kw):
    assert L.pi0_pages_workspace_bytes(ctypes.byref(good(**kw))) > 0


def test_page_operations_refuse(L):
    p = ctypes.byref(good())
    need = L.pi0_pages_workspace_bytes(p)
    assert L.pi0_pages_reserve(p, None, FAKE, need, None) == binding.PI0_EINVAL
    assert L.pi0_pages_reserve(p, FAKE, None, need, None) == binding.PI0_EINVAL
    assert L.pi0_pages_reserve(p, FAKE, FAKE + 8, need, None) == binding.PI0_EINVAL
    assert L.pi0_pages_reserve(p, FAKE, FAKE, need - 1, None) == binding.PI0_ENOMEM
    assert L.pi0_pages_compact(p, None, FAKE, -1, FAKE, FAKE, need, None) == binding.PI0_EINVAL
    assert L.pi0_pages_compact(p, None, None, 3, FAKE, FAKE, need, None) == binding.PI0_EINVAL
    assert L.pi0_pages_compact(p, None, FAKE, 3, None, FAKE, need, None) == binding.PI0_EINVAL
    assert L.pi0_pages_compact(p, None, FAKE, 3, FAKE, FAKE, need - 1, None) == binding.PI0_ENOMEM
    for n in (0, -1, 5):
        assert L.pi0_pages_fork(p, FAKE, FAKE, n, None) == binding.PI0_EINVAL
    assert L.pi0_pages_fork(p, None, FAKE, 1, None) == binding.PI0_EINVAL
    assert L.pi0_pages_fork(p, FAKE, None, 1, None) == binding.PI0_EINVAL


def rows(n, **kw):
    return binding.RowsC(**{**dict(d_x=FAKE, row_stride=n * 256, head_stride=256, heads=n, dtype=0), **kw})


BAD_ROWS = [dict(d_x=None), dict(d_x=FAKE + 8), dict(row_stride=248), dict(row_stride=2052), dict(head_stride=0), dict(head_stride=260), dict(heads=0),
            dict(heads=1025), dict(dtype=1)]


def test_norm_rope_refuses(L):
    ref = ctypes.byref

    def call(pages=good(), layer=0, q=rows(8), k=rows(1), v=rows(1), out=rows(8), starts=FAKE, n=3, most=3, pos=None, qg=None, kg=None, eps=1e-6,
             dim=256, base=1e4):
        return L.pi0_qk_norm_rope(ref(pages), layer, q and ref(q), k and ref(k), v and ref(v), out and ref(out), starts, n, most, pos, qg, kg, 1.0,
                                  eps, dim, base, 0, None)
    bad = [dict(layer=-1), dict(layer=18), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(k=rows(2)), dict(v=rows(2)), dict(out=rows(4)),
           dict(starts=None), dict(starts=FAKE + 2), dict(n=0), dict(most=0), dict(most=4), dict(n=(1 << 24) + 1), dict(pos=FAKE + 1), dict(qg=FAKE + 4),
           dict(kg=FAKE + 4), dict(eps=-1.0), dict(eps=float("nan")), dict(dim=-8), dict(dim=4), dict(dim=264), dict(base=0.0), dict(base=float("inf")),
           dict(q=rows(8, dtype=2)), dict(q=rows(8, dtype=2), k=rows(1, dtype=2), v=rows(1, dtype=2), out=rows(8, dtype=2)), dict(pages=good(dtype=1))]
    bad += [dict(q=rows(8, **kw)) for kw in BAD_ROWS] + [dict(out=rows(8, **kw)) for kw in BAD_ROWS] + [dict(pages=good(**kw)) for kw in BAD_PAGES]
    for kw in bad:
        assert call(**kw) == binding.PI0_EINVAL, {k: v for k, v in kw.items()}


def test_tree_attention_refuses(L):
    ref = ctypes.byref
    need = L.pi0_tree_attention_workspace_bytes(ref(good()), 8, 3, 3)
    assert need > 0

    def call(pages=good(), layer=0, q=rows(8), out=rows(8), starts=FAKE, n=3, most=3, mask=FAKE, words=1, scale=0.1, ws=FAKE, size=need):
        return L.pi0_tree_attention(ref(pages), layer, q and ref(q), out and ref(out), starts, n, most, mask, words, scale, ws, size, None)
    bad = [dict(layer=-1), dict(layer=18), dict(q=None), dict(out=None), dict(out=rows(4)), dict(starts=None), dict(starts=FAKE + 2), dict(n=0), dict(most=0),
           dict(most=4), dict(n=2000, most=1025), dict(mask=None), dict(words=0), dict(words=-1), dict(words=33), dict(mask=FAKE + 1), dict(ws=None), dict(ws=FAKE + 8),
           dict(scale=float("inf")), dict(scale=float("nan")), dict(pages=good(dtype=1)), dict(pages=good(kv_heads=3, token_stride=3 * 256, page_stride=64 * 3 * 256,
                                                                                                    layer_stride=640 * 3 * 256))]
    bad += [dict(q=rows(8, **kw)) for kw in BAD_ROWS] + [dict(out=rows(8, **kw)) for kw in BAD_ROWS] + [dict(pages=good(**kw)) for kw in BAD_PAGES]
    for kw in bad:
        assert call(**kw) == binding.PI0_EINVAL, kw
    assert call(size=need - 1) == binding.PI0_ENOMEM


def test_strides_and_lines_at_their_limits(L):
    """Rows 2^27 elements apart, and as many granules of all units together as 2^30, are refused; one step below is taken."""
    ref = ctypes.byref
    far = dict(token_stride=1 << 27, page_stride=1 << 34, layer_stride=1 << 38, layers=2, n_pages=2)
    near = dict(far, token_stride=(1 << 27) - 8)
    assert L.pi0_tree_attention_workspace_bytes(ref(good(**far)), 8, 1, 1) == 0 and L.pi0_pages_workspace_bytes(ref(good(**far))) == 0
    assert L.pi0_tree_attention_workspace_bytes(ref(good(**near)), 8, 1, 1) > 0
    # 1024 sequences, 8 tiles of 16 rows (128 of one key/value head): 2^17 granules and 6 more each are too many, half of that is not
    wide = dict(n_seqs=1024, page_tokens=256, max_pages=1 << 14, page_stride=256 * 256, layer_stride=10 * 256 * 256)
    assert L.pi0_tree_attention_workspace_bytes(ref(good(**wide)), 8, 2048, 16) == 0
    assert L.pi0_tree_attention_workspace_bytes(ref(good(**dict(wide, max_pages=1 << 13))), 8, 2048, 16) > 0
    # one tile: 2^20 * 1024 positions would pass it too, but a list is shorter than that
    assert L.pi0_tree_attention_workspace_bytes(ref(good(**dict(wide, max_pages=1 << 16))), 8, 2, 1) > 0


def test_store_and_load_refuse(L):
    cfg = synth.reduced_config()
    ctx = ctypes.c_void_p()
    assert L.pi0_create(ctypes.byref(binding.to_c_config(cfg)), ctypes.byref(ctx)) == 0
    mine = dict(layers=cfg.llm_layers)
    for kw in (dict(layers=3), dict(kv_heads=2, token_stride=512, page_stride=64 * 512, layer_stride=640 * 512), dict(head_dim=128), dict(dtype=1), dict(d_k=None)):
        p = ctypes.byref(good(**{**mine, **kw}))
        assert L.pi0_pages_store(ctx, p, 0, None) == binding.PI0_EINVAL, kw
        assert L.pi0_pages_load(ctx, p, 0, 256, None) == binding.PI0_EINVAL, kw
    p = ctypes.byref(good(**mine))
    for seq in (-1, 4):
        assert L.pi0_pages_store(ctx, p, seq, None) == binding.PI0_EINVAL and L.pi0_pages_load(ctx, p, seq, 256, None) == binding.PI0_EINVAL
    for n in (0, 255, 3 * 256 + 49):
        assert L.pi0_pages_load(ctx, p, 0, n, None) == binding.PI0_EINVAL
    assert L.pi0_pages_store(None, p, 0, None) == binding.PI0_EINVAL and L.pi0_pages_load(None, p, 0, 256, None) == binding.PI0_EINVAL
    # no weights, no prefill
    assert L.pi0_pages_store(ctx, p, 0, None) == binding.PI0_ESTATE and L.pi0_pages_load(ctx, p, 0, 256, None) == binding.PI0_ESTATE
    assert L.pi0_last_hip_error(ctx) == 0
    L.pi0_destroy(ctx)


def test_binding_refuses_tensors_of_other_kinds(L):
    k = torch.zeros((2, 6, 16, 1, 64), dtype=torch.bfloat16)
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    for args in ((k, k, i(3, 2), i(3), i(6)),                                   # not on a GPU
                 (k, k[:1], i(3, 2), i(3), i(6)), (k.float(), k, i(3, 2), i(3), i(6)), (k, k.transpose(1, 2).contiguous().transpose(1, 2), i(3, 2), i(3), i(6)),
                 (k, k, i(3, 2).long(), i(3), i(6)), (k, k, i(3, 2), i(4), i(6)), (k, k, i(3, 2), i(3), i(5)), (k, k, i(2, 3).t(), i(3), i(6))):
        with pytest.raises(binding.Pi0Error) as e:
            binding.Pages(*args)
        assert e.value.code == binding.PI0_EINVAL


# ------------------------------------------------------------------------------------- the plain bookkeeping, pinned
def contents(c, s):
    return [tuple(pool[layer, page, row].tolist() for pool in (c.k, c.v) for layer in range(c.k.shape[0]))
            for page, row in (c.place(s, pos) for pos in range(c.length[s]))]


def test_plain_cache_keeps_what_its_sequences_hold():
    """Random operations: a sequence's contents are a list on which the operations are what they are on lists, the reference
    counts are how often a page is listed, and a refused operation changes nothing."""
    rng = np.random.default_rng(5)
    pools = rng.standard_normal((2, 2, 40, 4, 1)).astype(np.float32)
    c = paged.Cache(pools[0], pools[1], 5, 12)
    want = [[] for _ in range(5)]
    refused = 0
    for step in range(400):
        s, kind = int(rng.integers(5)), int(rng.integers(4))
        before = copy.deepcopy((c.table, c.length, c.refs))
        values = [x.copy() for x in (c.k, c.v)]
        try:
            if kind <= 1:          # draft a few tokens and accept some of them
                n = int(rng.integers(0, 9))
                c.reserve([n if i == s else -1 for i in range(5)])
                drafts = rng.standard_normal((n, 4)).astype(np.float32)
                for j in range(n):
                    page, row = c.place(s, c.length[s] + j)
                    assert c.refs[page] == 1
                    c.k[:, page, row, 0], c.v[:, page, row, 0] = drafts[j, :2], drafts[j, 2:]
                keep = np.flatnonzero(rng.random(n) < 0.6)
                c.compact([keep] * 5, [len(keep) if i == s else -1 for i in range(5)])
                want[s] = want[s] + [tuple([float(x)] for x in drafts[j]) for j in keep]
            elif kind == 2:
                d = int(rng.integers(5))
                c.fork([s], [d])
                want[d] = list(want[s])
            else:
                start = int(rng.integers(0, c.length[s] + 1))
                keep = np.flatnonzero(rng.random(c.length[s] - start) < rng.random())
                c.compact([keep] * 5, [len(keep) if i == s else -1 for i in range(5)], [start] * 5 if start <= min(c.length) else [start if i == s else 0 for i in range(5)])
                want[s] = want[s][:start] + [want[s][start + j] for j in keep]
        except paged.Refused:
            refused += 1
            assert (c.table, c.length, c.refs) == before or kind <= 1
            if kind > 1:
                assert np.array_equal(values[0], c.k) and np.array_equal(values[1], c.v)
        assert [contents(c, i) for i in range(5)] == want, step
        assert c.refs == [sum(t.count(p) for t in c.table) for p in range(40)]
    assert 0 < refused < 300


def test_plain_norm_rope_keeps_lengths_and_relative_positions():
    rng = np.random.default_rng(6)
    x = rng.standard_normal((3, 2, 64))
    for inter in (False, True):
        y = paged.norm_rope(x, None, 0.0, 0.0, [0, 5, 70000], 64, 1e4, inter)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(y[0], x[0])
        dot = [(paged.norm_rope(x[:1], None, 0, 0, [p], 64, 1e4, inter) * paged.norm_rope(x[1:2], None, 0, 0, [p + 9], 64, 1e4, inter)).sum() for p in (0, 300)]
        assert abs(dot[0] - dot[1]) < 1e-9
        z = paged.norm_rope(x, np.zeros(64), 1.0, 0.0, [0, 0, 0], 0, 1e4, inter)
        assert np.allclose((z ** 2).mean(-1), 1.0)


def test_plain_attention_against_torch():
    rng = np.random.default_rng(7)
    q, k, v = rng.standard_normal((5, 4, 8)), rng.standard_normal((9, 2, 8)), rng.standard_normal((9, 2, 8))
    seen = rng.random((5, 9)) < 0.5
    seen[2] = False
    got = paged.attention(q, k, v, seen, 0.3)
    t = [torch.from_numpy(x).transpose(0, 1) for x in (q, np.repeat(k, 2, 1), np.repeat(v, 2, 1))]
    want = torch.nn.functional.scaled_dot_product_attention(*t, attn_mask=torch.from_numpy(seen), scale=0.3).transpose(0, 1).numpy()
    alive = [0, 1, 3, 4]
    assert np.allclose(got[alive], want[alive]) and not got[2].any()


def test_layers_that_one_launch_can_move(L):
    """A move has a block of 256 threads per 128 elements of a layer's keys and of its values: more than fit one launch are refused, at the
    door and not behind the plan."""
    def wide(**kw):
        c = dict(kv_heads=256, head_dim=256, token_stride=1 << 16, page_stride=1 << 20, page_tokens=16, n_pages=1, layers=1 << 13, layer_stride=1 << 20)
        return ctypes.byref(good(**{**c, **kw}))
    assert L.pi0_pages_workspace_bytes(wide()) > 0
    for kw in (dict(layers=(1 << 13) + 1), dict(layers=1 << 16), dict(layers=(1 << 16) + 1, kv_heads=1, head_dim=64)):
        assert L.pi0_pages_workspace_bytes(wide(**kw)) == 0, kw
        assert L.pi0_pages_reserve(wide(**kw), FAKE, FAKE, 1 << 40, None) == binding.PI0_EINVAL
        assert L.pi0_pages_compact(wide(**kw), None, FAKE, 1, FAKE, FAKE, 1 << 40, None) == binding.PI0_EINVAL
    # the grid of the largest that is taken: blocks of 128 elements, keys and values
    assert (1 << 29) // 128 * 2 * 256 + 2 * 256 * (1 << 16) < 1 << 32


def cache_without_a_gpu(**kw):
    """What the checks of arguments look at, of a cache whose tensors are on no GPU."""
    p = object.__new__(binding.Pages)
    p._c = good(**{**dict(n_seqs=2), **kw})
    p._ref, p.n_seqs, p.device, p._index, p._streams = ctypes.byref(p._c), 2, torch.device("cuda:0"), 0, set()
    return p


def test_a_mask_of_no_words_is_not_no_mask(L):
    """Rows that would see no drafted token at all are not taken for rows that see all up to themselves."""
    p = cache_without_a_gpu()
    p._on = lambda *a: pytest.fail("taken")
    q, starts = torch.zeros((3, 8, 256), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(binding.Pi0Error) as e:
        binding.pi0_tree_attention(p, 0, q, starts, 2, mask=torch.zeros((3, 0), dtype=torch.int32))
    assert e.value.code == binding.PI0_EINVAL


def test_a_scale_that_overflows(L):
    """The kernel takes scale * log2(e): where that is infinite, scores of zero would become NaN."""
    ref = ctypes.byref
    need = L.pi0_tree_attention_workspace_bytes(ref(good()), 8, 3, 3)
    for scale in (2.0 ** 127, -2.0 ** 127, 3e38, -3.4e38):
        assert L.pi0_tree_attention(ref(good()), 0, ref(rows(8)), ref(rows(8)), FAKE, 3, 3, None, 0, scale, FAKE, need, None) == binding.PI0_EINVAL, scale


def test_strides_of_a_single_row_or_head_say_nothing(L):
    """A token's queries out of a fused row of odd width, a head whose axis has stride 1."""
    ref = ctypes.byref
    fused = torch.zeros((5, 10 * 64 + 3), dtype=torch.bfloat16)
    one = fused[2:3, :512].unflatten(1, (8, 64))
    r = binding._rows(one, "q", 1, 8, 64)
    assert r.row_stride % 8 == 0 and r.row_stride >= 64 and r.head_stride == 64 and r.d_x == one.data_ptr()
    head = torch.zeros((3, 64, 1), dtype=torch.bfloat16).transpose(1, 2)
    assert head.stride(1) == 1 and binding._rows(head, "q", 3, 1, 64).head_stride == 64
    k = torch.zeros((2, 5, 16, 64, 1), dtype=torch.bfloat16).transpose(3, 4)
    assert k.stride(3) == 1 and binding._strides(k) == [5 * 16 * 64, 16 * 64, 64, 0]
    p = good(layers=2, n_pages=5, page_tokens=16, head_dim=64)
    p.layer_stride, p.page_stride, p.token_stride, p.head_stride = binding._strides(k)
    assert L.pi0_pages_workspace_bytes(ref(p)) > 0


def test_the_reciprocal_finds_a_rows_token():
    """Attention finds row r's token as (r + 1/2) * reciprocal(group) in fp32, cut off.  At the first and last row of every token, for every group up to
    1024 and 1024 tokens, with a reciprocal one step to either side of the rounded one, as far off as the hardware's may be."""
    token = np.arange(1024, dtype=np.int64)
    for group in range(1, 1025):
        near = np.float32(1.0) / np.float32(group)
        for reciprocal in (np.nextafter(near, np.float32(0)), near, np.nextafter(near, np.float32(2))):
            for row in (token * group, token * group + group - 1):
                found = ((row.astype(np.float32) + np.float32(0.5)) * np.float32(reciprocal)).astype(np.int64)
                assert np.array_equal(found, token), group
