"""GPU: reserve, fork and compact against the plain bookkeeping, whole pools and tables bit for bit, over layouts, page sizes
and the calls that the device refuses."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2510_26742_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def say(*a):
    print(*a, flush=True)


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def make(seed, layers=3, n_pages=40, page=16, kv_heads=1, head_dim=64, n_seqs=6, max_pages=9, order=(0, 1, 2, 3), dtype=torch.bfloat16):
    """The same empty cache twice: on the GPU, with the axes before head_dim stored in `order`, and as plain arrays of its bits."""
    shape = (layers, n_pages, page, kv_heads)
    g = torch.Generator().manual_seed(seed)
    pools = []
    for _ in range(2):
        t = torch.empty([shape[i] for i in order] + [head_dim], dtype=dtype, device=DEV).permute(*[order.index(i) for i in range(4)], 4)
        t.copy_(torch.randn((*shape, head_dim), generator=g))
        pools.append(t)
    gpu = binding.Pages(*pools, ints(np.full((n_seqs, max_pages), -1)), ints(np.zeros(n_seqs)), ints(np.zeros(n_pages)))
    return gpu, paged.Cache(*[bits(t) for t in pools], n_seqs, max_pages)


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().copy()


def same(gpu, cpu, where=""):
    torch.cuda.synchronize()
    np.testing.assert_array_equal(gpu.table.cpu().numpy(), cpu.table_array(), err_msg=f"table {where}")
    np.testing.assert_array_equal(gpu.length.cpu().numpy(), cpu.length, err_msg=f"length {where}")
    np.testing.assert_array_equal(gpu.refs.cpu().numpy(), cpu.refs, err_msg=f"refs {where}")
    for name in ("k", "v"):
        np.testing.assert_array_equal(bits(getattr(gpu, name)), getattr(cpu, name), err_msg=f"{name} {where}")


def grow(gpu, cpu, lengths):
    """Sequences of these lengths, holding what their pages hold."""
    gpu.pi0_pages_reserve(ints(lengths))
    cpu.reserve(lengths)
    keep = [list(range(n)) for n in lengths]
    wide = np.zeros((len(lengths), max(1, max(lengths))))
    for s, row in enumerate(keep):
        wide[s, :len(row)] = row
    gpu.pi0_pages_compact(ints(wide), ints(lengths))
    cpu.compact(keep, lengths)
    gpu.pi0_pages_status()


@pytest.mark.parametrize("kw", [dict(), dict(kv_heads=3, head_dim=128, page=32, order=(0, 1, 3, 2)), dict(order=(1, 2, 0, 3), kv_heads=2, n_seqs=40, n_pages=90, max_pages=70),
                                dict(layers=1, head_dim=256, page=64, kv_heads=2, dtype=torch.float16), dict(page=256, n_pages=9, n_seqs=3, max_pages=3),
                                dict(layers=2, kv_heads=20, head_dim=64, order=(3, 1, 2, 0)), dict(n_pages=2500, n_seqs=200, max_pages=20, layers=1)])
def test_random_operations(kw):
    say("[gpu] pages", kw)
    gpu, cpu = make(1, **kw)
    rng = np.random.default_rng(2)
    n_seqs, most = len(cpu.table), cpu.max_pages * cpu.page
    refused = 0
    for step in range(30):
        kind = int(rng.integers(3))
        snapshot = (cpu.table_array(), list(cpu.length), list(cpu.refs))
        try:
            if kind == 0:
                extra = [int(rng.integers(-1, 30)) if rng.random() < 0.7 else -1 for _ in range(n_seqs)]
                if rng.random() < 0.1:
                    extra[int(rng.integers(n_seqs))] = most + 1
                gpu.pi0_pages_reserve(ints(extra))
                cpu.reserve(extra)
            elif kind == 1:
                n = int(rng.integers(1, max(2, n_seqs // 2)))
                who = rng.permutation(n_seqs)
                src, dst = [int(x) for x in rng.choice(who[:n], n)], [int(x) for x in who[n:2 * n]]
                src = src[:len(dst)]
                if rng.random() < 0.2:
                    dst[-1] = [src[0], dst[0], -1, n_seqs][int(rng.integers(4))]
                gpu.pi0_pages_fork(ints(src), ints(dst))
                cpu.fork(src, dst)
            else:
                start, keep, n_keep = [], np.zeros((n_seqs, most), dtype=np.int64), []
                for s in range(n_seqs):
                    room = len(cpu.table[s]) * cpu.page
                    start.append(int(rng.integers(0, cpu.length[s] + 1)) if rng.random() < 0.4 else cpu.length[s])
                    mine = np.flatnonzero(rng.random(room - start[s]) < rng.random())[:most]
                    if rng.random() < 0.3:
                        mine = np.arange(min(len(mine), 5))
                    keep[s, :len(mine)] = mine
                    n_keep.append(len(mine) if rng.random() < 0.8 else -1)
                if rng.random() < 0.15 and max(n_keep) > 0:
                    s = int(np.argmax(n_keep))
                    keep[s, n_keep[s] - 1] = [-1, most, 0 if n_keep[s] > 1 else -5][int(rng.integers(3))]
                gpu.pi0_pages_compact(ints(keep), ints(n_keep), start=ints(start))
                cpu.compact(keep, n_keep, start)
            gpu.pi0_pages_status()
        except paged.Refused as e:
            refused += 1
            with pytest.raises(binding.Pi0Error) as got:
                gpu.pi0_pages_status()
            assert got.value.code == (binding.PI0_ENOMEM if "room" in str(e) else binding.PI0_EINVAL)
            cpu.table = [[int(p) for p in row if p >= 0] for row in snapshot[0]]
            cpu.length, cpu.refs = snapshot[1], snapshot[2]
        same(gpu, cpu, f"step {step} kind {kind}")
    assert refused < 25


def test_long_compaction_in_place_and_into_own_pages():
    gpu, cpu = make(3, layers=2, n_pages=200, page=32, kv_heads=2, head_dim=128, n_seqs=3, max_pages=64)
    grow(gpu, cpu, [1900, 0, 333])
    gpu.pi0_pages_fork(ints([0]), ints([1]))
    cpu.fork([0], [1])
    rng = np.random.default_rng(4)
    keep = np.zeros((3, 1900), dtype=np.int64)
    n_keep = []
    for s, n in enumerate(cpu.length):
        mine = np.flatnonzero(rng.random(n) < 0.7)
        keep[s, :len(mine)] = mine
        n_keep.append(len(mine))
    # the fork alone (its source keeps the pages), then its source and the third in place
    for who in ([-1, n_keep[1], -1], [n_keep[0], -1, n_keep[2]]):
        gpu.pi0_pages_compact(ints(keep), ints(who), start=ints([0, 0, 0]))
        cpu.compact(keep, who, [0, 0, 0])
        gpu.pi0_pages_status()
        same(gpu, cpu)


@pytest.mark.parametrize("first", [0, 63, 511, 512, 1030, 1500])
def test_lists_and_choices_of_more_than_one_read(first):
    """119 and more pages, shared by three, of which positions from `first` on close up: shared pages in front of and behind a
    list's 64th entry are replaced, others not; then a reservation behind them; then a choice with one mistake far behind."""
    gpu, cpu = make(9, layers=1, n_pages=600, page=16, kv_heads=1, head_dim=64, n_seqs=4, max_pages=150)
    grow(gpu, cpu, [1900, 0, 0, 40])
    gpu.pi0_pages_fork(ints([0, 0]), ints([1, 2]))
    cpu.fork([0, 0], [1, 2])
    keep = [i for i in range(1900) if i < first or i % 3][:1600]
    table = np.zeros((4, 1600))
    table[0, :len(keep)] = keep
    table[2, :5] = [0, 1, 2, 3, 900]
    n, start = [len(keep), -1, 5, -1], [0, 1900, 1000, 40]
    gpu.pi0_pages_compact(ints(table), ints(n), start=ints(start))
    cpu.compact(table.astype(int), n, start)
    same(gpu, cpu, "compacted")
    gpu.pi0_pages_reserve(ints([300, 1, 20, 0]))
    cpu.reserve([300, 1, 20, 0])
    same(gpu, cpu, "reserved")
    table[1, :1600] = np.arange(1600)
    table[1, 1333] = 1332
    gpu.pi0_pages_compact(ints(table), ints([-1, 1600, -1, -1]), start=ints([0] * 4))
    with pytest.raises(binding.Pi0Error):
        gpu.pi0_pages_status()
    same(gpu, cpu, "refused")


def test_everything_can_be_freed_and_lengths_start_at_nothing():
    gpu, cpu = make(5)
    zero = [0] * 6
    gpu.pi0_pages_reserve(ints(zero))
    cpu.reserve(zero)
    gpu.pi0_pages_compact(None, ints(zero))
    cpu.compact(None, zero)
    gpu.pi0_pages_fork(ints([0, 0]), ints([1, 2]))      # of an empty sequence
    cpu.fork([0, 0], [1, 2])
    gpu.pi0_pages_status()
    same(gpu, cpu)
    grow(gpu, cpu, [17, 16, 1, 0, 48, 15])
    same(gpu, cpu)
    gpu.pi0_pages_compact(None, ints(zero), start=ints(zero))
    cpu.compact(None, zero, zero)
    gpu.pi0_pages_status()
    same(gpu, cpu)
    assert not cpu.refs.count(1) and int(gpu.refs.sum()) == 0


def test_status_is_told_once_and_nothing_is_changed():
    gpu, cpu = make(6, n_pages=4)
    with pytest.raises(binding.Pi0Error) as e:
        gpu.pi0_pages_reserve(ints([16, 16, 16, 16, 1, -1]))     # five pages
        gpu.pi0_pages_status()
    assert e.value.code == binding.PI0_ENOMEM
    gpu.pi0_pages_status()
    same(gpu, cpu)
    for src, dst in (([0], [0]), ([0, 1], [2, 2]), ([0], [6]), ([-1], [0]), ([0, 1], [1, 2])):
        gpu.pi0_pages_fork(ints(src), ints(dst))
        with pytest.raises(binding.Pi0Error) as e:
            gpu.pi0_pages_status()
        assert e.value.code == binding.PI0_EINVAL
        same(gpu, cpu)


def test_tables_with_entries_that_are_no_pages():
    """A list ends where its entries stop being pages; what does not fit it is refused."""
    gpu, cpu = make(7)
    grow(gpu, cpu, [20, 0, 0, 0, 0, 0])
    gpu.table[0, 2:5] = ints([1 << 30, -7, 40])                 # 40: one behind the last page
    cpu.table[0] = cpu.table[0][:2]
    gpu.pi0_pages_reserve(ints([13, -1, -1, -1, -1, -1]))       # 33 positions: one page more, in place of what is no page
    cpu.reserve([13] + [-1] * 5)
    gpu.pi0_pages_status()
    gpu.table[0, 3:5] = -1
    same(gpu, cpu)
    gpu.length[1] = 5                                          # committed, but no page
    gpu.pi0_pages_fork(ints([1]), ints([2]))
    with pytest.raises(binding.Pi0Error):
        gpu.pi0_pages_status()
    gpu.pi0_pages_reserve(ints([-1, 0, -1, -1, -1, -1]))
    with pytest.raises(binding.Pi0Error):
        gpu.pi0_pages_status()
    gpu.length[1] = 0
    same(gpu, cpu)


def test_captured_and_replayed_beside_eager_calls():
    """One graph of reserve, compact and fork, replayed with other numbers in the same tensors, on a stream of its own."""
    gpu, cpu = make(8, n_pages=60)
    grow(gpu, cpu, [30, 10, 0, 0, 0, 0])
    stream = torch.cuda.Stream()
    extra, keep, n_keep, src, dst = ints([4] * 6), ints(np.zeros((6, 4))), ints([0] * 6), ints([0]), ints([2])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        gpu.pi0_pages_reserve(extra, stream=stream)
        gpu.pi0_pages_compact(keep, n_keep, stream=stream)
        gpu.pi0_pages_fork(src, dst, stream=stream)
    rng = np.random.default_rng(9)
    for step in range(6):
        say("[gpu] replay", step)
        e = [int(x) for x in rng.integers(0, 5, 6)]
        rows = [np.flatnonzero(rng.random(n) < 0.6) for n in e]
        a, b = [int(x) for x in rng.permutation(6)[:2]]
        wide = np.zeros((6, 4), dtype=np.int64)
        for s, r in enumerate(rows):
            wide[s, :len(r)] = r
        for t, x in ((extra, e), (keep, wide), (n_keep, [len(r) for r in rows]), (src, [a]), (dst, [b])):
            t.copy_(ints(x))
        torch.cuda.synchronize()
        graph.replay()
        cpu.reserve(e)
        cpu.compact(rows, [len(r) for r in rows])
        cpu.fork([a], [b])
        torch.cuda.synchronize()
        gpu.pi0_pages_status()
        same(gpu, cpu, f"replay {step}")
        gpu.pi0_pages_compact(None, ints([-1] * 5 + [0]), start=ints([0] * 6))      # eager, in between
        cpu.compact(None, [-1] * 5 + [0], [0] * 6)
        same(gpu, cpu, f"eager {step}")


def hip_error_left(code=12345):
    """An error that a call of the caller's own left in this thread (a device that is none), and the runtime's way to fetch it."""
    import ctypes
    hip = ctypes.CDLL(binding.LIB_PATH)
    hip.hipSetDevice.argtypes, hip.hipSetDevice.restype = [ctypes.c_int], ctypes.c_int
    hip.hipGetLastError.restype = ctypes.c_int
    assert hip.hipSetDevice(code) != 0
    return hip.hipGetLastError


def test_an_error_left_by_the_caller_is_not_a_calls_own():
    """Both halves of reserve and compact run, and every call says PI0_OK, although the thread's last error is another call's."""
    gpu, cpu = make(10, layers=2, kv_heads=2)
    grow(gpu, cpu, [40, 5, 0, 0, 0, 0])
    src, dst, extra, n, start = ints([0]), ints([2]), ints([-1, -1, 3, -1, -1, -1]), ints([20, -1, -1, -1, -1, -1]), ints([0] * 6)
    keep = ints([[2 * i for i in range(20)]] * 6)
    ws = torch.empty(gpu._plan_bytes, dtype=torch.uint8, device=DEV)
    q, k = torch.ones((1, 2, 64), dtype=torch.bfloat16, device=DEV), torch.ones((1, 2, 64), dtype=torch.bfloat16, device=DEV)
    starts = ints([0, 1, 1, 1, 1, 1, 1])
    rows = binding._rows(q, "q", 1, 2, 64)
    room = binding.lib().pi0_tree_attention_workspace_bytes(gpu._ref, 2, 1, 1)
    ws2, out = torch.empty(room, dtype=torch.uint8, device=DEV), torch.empty_like(q)
    torch.cuda.synchronize()
    L, ref, last = binding.lib(), gpu._ref, hip_error_left
    calls = [lambda: L.pi0_pages_fork(ref, src.data_ptr(), dst.data_ptr(), 1, None),
             lambda: L.pi0_pages_reserve(ref, extra.data_ptr(), ws.data_ptr(), gpu._plan_bytes, None),
             lambda: L.pi0_pages_compact(ref, start.data_ptr(), keep.data_ptr(), 20, n.data_ptr(), ws.data_ptr(), gpu._plan_bytes, None)]
    codes = []
    for call in calls:
        fetch = last()
        codes.append(call())
        fetch()
    assert codes == [binding.PI0_OK] * 3
    torch.cuda.synchronize()
    cpu.fork([0], [2])
    cpu.reserve([-1, -1, 3, -1, -1, -1])
    cpu.compact([[2 * i for i in range(20)]] * 6, [20, -1, -1, -1, -1, -1], [0] * 6)
    gpu.pi0_pages_status()
    same(gpu, cpu)
    gpu.pi0_pages_reserve(ints([1, -1, -1, -1, -1, -1]))
    import ctypes
    r, o = ctypes.byref(rows), ctypes.byref(binding._rows(out, "out", 1, 2, 64))
    kr = ctypes.byref(binding._rows(k, "k", 1, 2, 64))
    for call in (lambda: L.pi0_qk_norm_rope(ref, 0, r, kr, kr, o, starts.data_ptr(), 1, 1, None, None, None, 1.0, 1e-6, 64, 1e4, 0, None),
                 lambda: L.pi0_tree_attention(ref, 0, r, o, starts.data_ptr(), 1, 1, None, 0, 0.125, ws2.data_ptr(), room, None)):
        fetch = last()
        code = call()
        fetch()
        assert code == binding.PI0_OK
    torch.cuda.synchronize()
    assert torch.isfinite(out.float()).all()


@pytest.mark.parametrize("inside", [True, False])
def test_what_a_call_was_given_stays_until_it_has_run(inside):
    """Tensors of the default stream, given to a call on another (which is torch's current one, or is not) and dropped: while that stream has not
    come to the call, their memory is not handed out again."""
    gpu, cpu = make(11)
    grow(gpu, cpu, [30, 30, 0, 0, 0, 0])
    side = torch.cuda.Stream()
    big = 300_001                                                     # a size that nothing else asks for
    keep = torch.zeros((6, big), dtype=torch.int32, device=DEV)
    keep[0, :10] = torch.arange(0, 20, 2, device=DEV)
    n, start = ints([10] + [-1] * 5), ints([0] * 6)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
    if inside:
        with torch.cuda.stream(side):
            gpu.pi0_pages_compact(keep, n, start=start, stream=side)
    else:
        gpu.pi0_pages_compact(keep, n, start=start, stream=side)
    where = keep.data_ptr()
    del keep
    other = torch.empty((6, big), dtype=torch.int32, device=DEV)
    busy = not side.query()
    assert busy and other.data_ptr() != where
    side.synchronize()
    cpu.compact([list(range(0, 20, 2))] * 6, [10] + [-1] * 5, [0] * 6)
    gpu.pi0_pages_status()
    same(gpu, cpu)


def test_free_pages_far_behind_others():
    """50 000 pages that others hold in front of the first free ones, which lie one by one and in runs across the reads of a search."""
    gpu, cpu = make(12, layers=1, n_pages=53_000, page=16, kv_heads=1, head_dim=64, n_seqs=3, max_pages=1200)
    taken = np.ones(53_000, dtype=np.int64)
    free = np.concatenate([[3, 1023, 1024], [50_000, 50_175, 50_176], np.arange(51_190, 51_700), [52_999], np.arange(52_000, 52_990)])
    taken[free] = 0
    gpu.refs.copy_(ints(taken))
    cpu.refs = taken.tolist()
    for extra in ([20, 50, -1], [16 * 5, -1, 16 * 700], [16 * 200, 3, 0]):
        gpu.pi0_pages_reserve(ints(extra))
        cpu.reserve(extra)
        gpu.pi0_pages_compact(ints([[0, 1, 2, 3]] * 3), ints([min(e, 4) for e in extra]))
        cpu.compact([[0, 1, 2, 3]] * 3, [min(e, 4) for e in extra])
        gpu.pi0_pages_status()
        same(gpu, cpu, str(extra))
    gpu.pi0_pages_reserve(ints([16 * 600, 16 * 600, 16 * 600]))
    with pytest.raises(paged.Refused):
        cpu.reserve([16 * 600] * 3)
    with pytest.raises(binding.Pi0Error) as e:
        gpu.pi0_pages_status()
    assert e.value.code == binding.PI0_ENOMEM
    same(gpu, cpu, "refused")


def test_as_many_sequences_as_there_can_be():
    """1024 sequences in every operation, half of them continuations of the other half, shared pages replaced for all at once."""
    gpu, cpu = make(13, layers=1, n_pages=5000, page=16, kv_heads=1, head_dim=64, n_seqs=1024, max_pages=4)
    rng = np.random.default_rng(14)
    grow(gpu, cpu, [int(x) for x in rng.integers(0, 40, 512)] + [0] * 512)
    src, dst = [int(x) for x in rng.integers(0, 512, 512)], [int(x) for x in 512 + rng.permutation(512)]
    gpu.pi0_pages_fork(ints(src), ints(dst))
    cpu.fork(src, dst)
    same(gpu, cpu, "forked")
    extra = [int(x) for x in rng.integers(-1, 17, 1024)]
    gpu.pi0_pages_reserve(ints(extra))
    cpu.reserve(extra)
    same(gpu, cpu, "reserved")
    start = [int(rng.integers(0, n + 1)) for n in cpu.length]
    rows = [np.flatnonzero(rng.random(len(t) * 16 - s) < 0.6) for t, s in zip(cpu.table, start)]
    keep, n = np.zeros((1024, 64), dtype=np.int64), []
    for s, r in enumerate(rows):
        keep[s, :len(r)] = r
        n.append(len(r) if s % 9 else -1)
    gpu.pi0_pages_compact(ints(keep), ints(n), start=ints(start))
    cpu.compact(keep, n, start)
    gpu.pi0_pages_status()
    same(gpu, cpu, "compacted")
