"""Group selection, ancestor masks and the append of accepted nodes against plain
forms (whole numbers: equal), the calls together as a speculative decoding step
makes them, on streams and in captured graphs."""
import numpy as np
import pytest
import torch

from tests import serving_ref as ref
from tests.test_gpu_canary import Guarded

pytestmark = pytest.mark.gpu
D = 128


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


@pytest.fixture(scope="module")
def ta(dev):
    import paper_2412_08585_amd as ta
    ta.lib()
    return ta


# ---- turbo_select_groups -------------------------------------------------------------
# Hq, bits, lengths, num_select, keep_first, keep_last
SELECTS = [
    (1, [4], [64], 1, 0, 0),
    (4, [4, 2], [0, 63, 64 * 3], 2, 1, 1),
    (8, [2], [64 * 9 + 5, 64 * 70], 5, 0, 2),
    (16, [4], [64 * 65], 64, 3, 4),
    (32, [2, 4], [64 * 300 + 1, 64 * 257, 64 * 256], 100, 1, 2),
    (10, [4, 2], [64 * 20], 30, 0, 0),           # more than there are
    (6, [2, 4, 4], [64 * 40, 64], 1, 1, 0),      # kept groups alone
    (4, [4, 2], [64 * 700 + 3, 64 * 513], 128, 1, 1),
    (2, [4], [64 * 1030], 40, 0, 3),             # bounds and choice in launches of their own
]


@pytest.mark.parametrize("case", range(len(SELECTS)))
def test_select_is_the_definition(ta, dev, case):
    Hq, bits, lens, num, first, last = SELECTS[case]
    print("select", SELECTS[case], flush=True)
    B = len(lens)
    f = ref.Filled(ta, dev, lens, bits, seed=case + 1).host()
    q = ref.rand((B, Hq, D), case)
    g = Guarded(dev)
    out = g((B, len(bits), num), torch.int32)
    ws = g((B * Hq * f.mg,), torch.float32)
    ta.turbo_select_groups(q.to(dev), f.cache, f.sl, f.btd, f.gtd, num, first, last, ws, out)
    g.check("turbo_select_groups")
    want = ref.select(f, q.numpy(), num, first, last)
    assert (out.cpu().numpy() == want).all()


def test_select_many_equal_scores(ta, dev):
    """70000 groups of three kinds: digit counts, ties and blocks past every width."""
    f = ref.Filled(ta, dev, [64 * 3], [4, 2], seed=5).host()
    mg = 70000
    rng = np.random.default_rng(1)
    f.mg, f.lens = mg, [64 * mg + 7]
    kind = rng.choice(3, size=mg, p=[0.001, 0.009, 0.99])
    f.gt = f.gt[0][kind][None].astype(np.int32)
    f.bt = f.bt[0].reshape(-1, 4)[kind].reshape(1, -1).astype(np.int32)
    f.gt[0, 5], f.bt[0, 4 * 69999] = -1, -1
    sl = torch.tensor(f.lens, dtype=torch.int32, device=dev)
    q = ref.rand((1, 4, D), 3)
    for num in (1, 50, 1000, 69999):
        got = ta.turbo_select_groups(q.to(dev), f.cache, sl, torch.from_numpy(f.bt).to(dev),
                                     torch.from_numpy(f.gt).to(dev), num, 1, 0)
        assert (got.cpu().numpy() == ref.select(f, q.numpy(), num, 1, 0)).all(), num


def test_select_many_heads_of_long_tables(ta, dev):
    """256 KV heads of 1100 groups (three kinds, over and over): one launch."""
    f = ref.Filled(ta, dev, [64 * 3], [4, 2] * 32, seed=6).host()
    mg, B = 1100, 4
    kind = np.random.default_rng(2).integers(0, 3, (B, mg))
    f.mg, f.lens = mg, [64 * mg, 64 * 900 + 5, 64 * 1025, 70]
    f.gt = f.gt[0][kind].astype(np.int32)
    f.bt = f.bt[0].reshape(-1, 4)[kind].reshape(B, -1).astype(np.int32)
    q = ref.rand((B, 64, D), 3)
    got = ta.turbo_select_groups(q.to(dev), f.cache, torch.tensor(f.lens, dtype=torch.int32, device=dev),
                                 torch.from_numpy(f.bt).to(dev), torch.from_numpy(f.gt).to(dev), 77, 1, 2)
    assert (got.cpu().numpy() == ref.select(f, q.numpy(), 77, 1, 2)).all()


def test_select_scores_that_are_no_numbers(ta, dev):
    """Scales of zero, infinity and NaN, a query of zeros, entries out of range."""
    f = ref.Filled(ta, dev, [64 * 40, 64 * 12], [4, 2], seed=7)
    for i, x in enumerate((0.0, float("inf"), float("nan"), -0.0)):
        f.cache.group_scale[f.gtd[0, 3 + i].long(), :, 0] = x
    f.cache.group_scale[f.gtd[1].long(), :, 0] = float("nan")
    f.bt[0, 4 * 20 + 2], f.bt[0, 4 * 21] = -1, f.cache.pages.shape[0]
    f.gt[0, 22], f.gt[0, 0], f.gt[0, 39] = f.cache.group_meta.shape[0], -1, -7
    f.btd.copy_(torch.from_numpy(f.bt))
    f.gtd.copy_(torch.from_numpy(f.gt))
    f.host()
    q = ref.rand((2, 8, D), 3)
    q[:, 1] = 0.0
    for num in (2, 9, 33, 38):
        got = ta.turbo_select_groups(q.to(dev), f.cache, f.sl, f.btd, f.gtd, num, 1, 1)
        assert (got.cpu().numpy() == ref.select(f, q.numpy(), num, 1, 1)).all(), num


# ---- turbo_tree_mask -----------------------------------------------------------------
@pytest.mark.parametrize("B,T", [(1, 1), (3, 16), (2, 63), (2, 64), (5, 65), (4, 200), (3, 256)])
def test_tree_mask(ta, dev, B, T):
    print("mask", B, T, flush=True)
    rng = np.random.default_rng(T)
    parents = np.stack([[rng.integers(-1, i) if i else -1 for i in range(T)] for _ in range(B)]).astype(np.int32)
    parents[0] = np.arange(T) - 1                     # a chain
    if B > 1:
        parents[1, T // 2:] = rng.integers(-9, T + 9, T - T // 2)  # later nodes, itself, outside: roots
    lens = rng.integers(0, T + 1, B)
    lens[0] = T + 3
    g = Guarded(dev)
    mask, depth = g((B, T, (T + 63) // 64), torch.int64), g((B, T), torch.int32)
    ta.turbo_tree_mask(torch.from_numpy(parents).to(dev),
                       torch.tensor(lens, dtype=torch.int32, device=dev), mask, depth)
    g.check("turbo_tree_mask")
    see, d = ref.ancestors(parents, lens)
    assert (mask.cpu().numpy() == ref.matrix_to_words(see)).all()
    assert (depth.cpu().numpy() == d).all()


# ---- turbo_append_path ---------------------------------------------------------------
# bits, lengths, T, max_path, path lengths
PATHS = [
    ([4], [64], 1, 1, [1]),
    ([4, 2], [0, 63, 64 * 3 + 60], 8, 6, [0, 6, 5]),
    ([2], [62, 64 * 2 + 1], 200, 200, [200, 190]),         # several buffers in one path
    ([2, 4, 4], [1, 64 * 4 - 1, -5, 64], 40, 64, [64, 1, 9, 99]),
]


def _clone(ta, f):
    """(cache, buffer) copies."""
    c = ta.PagedKVCache(1, 1, f.bits, "cpu")
    c.pages, c.group_meta, c.group_scale = (x.clone() for x in (f.cache.pages, f.cache.group_meta,
                                                                f.cache.group_scale))
    t = ta.KVTail(1, f.Hkv, "cpu")
    t.batch = f.tail.batch
    t.k, t.v, t.scale = f.tail.k.clone(), f.tail.v.clone(), f.tail.scale.clone()
    return c, t


def _one_by_one(ta, f, kt, vt, path, plen, cache, tail):
    """turbo_append_kv per node, sequence by sequence."""
    T = kt.shape[2]
    for b, n in enumerate(f.lens):
        p = n
        for i in range(min(max(plen[b], 0), path.shape[1])):
            node = int(path[b, i])
            if n < 0 or not 0 <= node < T:
                break
            ta.turbo_append_kv(kt[b:b + 1, :, node].contiguous(), vt[b:b + 1, :, node].contiguous(),
                               torch.tensor([p], dtype=torch.int32, device=kt.device), cache,
                               tail.narrow(b, 1), f.btd[b:b + 1], f.gtd[b:b + 1])
            p += 1


def _same_state(c, t, c2, t2):
    for x, y in ((c.pages, c2.pages), (c.group_meta, c2.group_meta), (c.group_scale, c2.group_scale),
                 (t.k, t2.k), (t.v, t2.v), (t.scale, t2.scale)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("case", range(len(PATHS)))
def test_append_path_is_one_append_per_node(ta, dev, case):
    bits, lens, T, P, plen = PATHS[case]
    print("path", PATHS[case], flush=True)
    B, Hkv = len(lens), len(bits)
    f = ref.Filled(ta, dev, lens, bits, seed=case + 21, max_groups=max(max(lens), 0) // 64 + 3)
    f.tail.scale.clamp_(min=0.02)  # (a sequence without tokens has no scale yet)
    kt, vt = ref.rand((B, Hkv, T, D), 1).to(dev), ref.rand((B, Hkv, T, D), 2).to(dev)
    kt[:, :, 0] *= 100  # codes that saturate
    rng = np.random.default_rng(case)
    path = rng.integers(0, T, (B, P)).astype(np.int32)  # nodes come up more than once
    if case == 3:
        path[0, 40], path[3, 2] = -1, T  # the path ends there
        f.gt[1, 3], f.bt[0, 1] = -1, f.cache.pages.shape[0]  # a group that cannot be written
        f.gtd.copy_(torch.from_numpy(f.gt))
        f.btd.copy_(torch.from_numpy(f.bt))
    want = _clone(ta, f)
    _one_by_one(ta, f, kt, vt, path, plen, *want)
    c, t = _clone(ta, f)
    g = Guarded(dev)
    for o in (c, t):
        for name in ("pages", "group_meta", "group_scale", "k", "v", "scale"):
            x = getattr(o, name, None)
            if x is not None:
                setattr(o, name, g(x.shape, x.dtype).copy_(x))
    ta.turbo_append_path(kt, vt, torch.from_numpy(path).to(dev),
                         torch.tensor(plen, dtype=torch.int32, device=dev), f.sl, c, t, f.btd, f.gtd)
    g.check("turbo_append_path")
    _same_state(c, t, *want)


def test_append_path_past_the_tables(ta, dev):
    """A buffer that fills up behind the last group of the table is not written."""
    f = ref.Filled(ta, dev, [64 * 2 + 50], [4, 2], seed=33, max_groups=2)
    kt, vt = ref.rand((1, 2, 30, D), 1).to(dev), ref.rand((1, 2, 30, D), 2).to(dev)
    path = np.arange(30, dtype=np.int32)[None]
    want = _clone(ta, f)
    _one_by_one(ta, f, kt, vt, path, [30], *want)
    c, t = _clone(ta, f)
    ta.turbo_append_path(kt, vt, torch.from_numpy(path).to(dev),
                         torch.tensor([30], dtype=torch.int32, device=dev), f.sl, c, t, f.btd, f.gtd)
    _same_state(c, t, *want)


# ---- together ------------------------------------------------------------------------
def _step(ta, f, q, kt, vt, parents, tl, path, plen, cache, tail, sl, bufs):
    """One drafted step: masks, attention, the accepted path, then a sparse decoding
    step of the first node's queries over the longer sequences."""
    mask, depth, o, lse, sel, o1, ws, wt, w1 = bufs
    ta.turbo_tree_mask(parents, tl, mask, depth)
    ta.turbo_attn_tree(q, kt, vt, mask, tl, cache, sl, f.btd, f.gtd, tail=tail, out=o, lse_out=lse,
                       workspace=wt)
    ta.turbo_append_path(kt, vt, path, plen, sl, cache, tail, f.btd, f.gtd)
    sl.add_(plen)
    q1 = q[:, :, 0].contiguous()
    ta.turbo_select_groups(q1, cache, sl, f.btd, f.gtd, sel.shape[2], 1, 1, ws, sel)
    ta.turbo_attn_selected(q1, cache, sl, f.btd, f.gtd, sel, tail=tail, out=o1, workspace=w1)


@pytest.fixture
def step(ta, dev):
    lens, bits, Hq, T, P = [64 * 6 + 60, 64 * 2 + 3, 63], [4, 2], 8, 24, 7
    B, Hkv = len(lens), len(bits)
    f = ref.Filled(ta, dev, lens, bits, seed=51, max_groups=10)
    rng = np.random.default_rng(3)
    parents = np.stack([[rng.integers(-1, i) if i else -1 for i in range(T)] for _ in range(B)]).astype(np.int32)
    see, depth = ref.ancestors(parents, [T] * B)
    path, plen = np.full((B, P), -1, np.int32), []
    for b in range(B):
        nodes = np.nonzero(see[b, depth[b].argmax()])[0][:P]
        path[b, :len(nodes)] = nodes
        plen.append(len(nodes))
    i32 = dict(dtype=torch.int32, device=dev)
    x = dict(f=f, q=ref.rand((B, Hq, T, D), 1).to(dev), kt=ref.rand((B, Hkv, T, D), 2).to(dev),
             vt=ref.rand((B, Hkv, T, D), 3).to(dev), parents=torch.tensor(parents, **i32),
             tl=torch.tensor([T] * B, **i32), path=torch.tensor(path, **i32),
             plen=torch.tensor(plen, **i32))

    def bufs():
        return (torch.zeros(B, T, 1, dtype=torch.int64, device=dev), torch.zeros(B, T, **i32),
                torch.zeros(B, Hq, T, D, dtype=torch.float16, device=dev),
                torch.zeros(B, Hq, T, device=dev), torch.zeros(B, Hkv, 4, **i32),
                torch.zeros(B, Hq, D, dtype=torch.float16, device=dev),
                ta.select_workspace(B, Hq, f.mg, dev),
                ta.tree_workspace(B, Hq, Hkv, T, f.mg, dev, with_tail=True),
                ta.selected_workspace(B, Hq, Hkv, 4, dev, with_tail=True))

    return x, bufs, see, plen


def test_a_drafted_step(ta, dev, step):
    """The calls together against their plain forms, over what each left."""
    x, bufs, see, plen = step
    f, out = x["f"], bufs()
    c, t = _clone(ta, f)
    want = _clone(ta, f)
    sl = f.sl.clone()
    from tests.test_gpu_attn_rows import _check, _check_tree
    _step(ta, **x, cache=c, tail=t, sl=sl, bufs=out)
    torch.cuda.synchronize()
    assert (out[0].cpu().numpy() == ref.matrix_to_words(see)).all()
    _check_tree(f, x["q"].cpu(), x["kt"].cpu(), x["vt"].cpu(), see, x["tl"].tolist(), out[2], out[3])
    _one_by_one(ta, f, x["kt"], x["vt"], x["path"].cpu().numpy(), plen, *want)
    _same_state(c, t, *want)
    f.cache, f.tail, f.lens = c, t, sl.tolist()
    f.host()
    q1 = x["q"][:, :, 0].cpu()
    assert (out[4].cpu().numpy() == ref.select(f, q1.numpy(), 4, 1, 1)).all()
    for b in range(f.B):
        for h in range(f.Hkv):
            kk, vv = f.kv(b, h, [g for g in out[4][b, h].tolist() if g >= 0])
            w, _, to, _ = ref.attend(q1[b, 4 * h:4 * h + 4].double().numpy(), kk, vv)
            _check(out[5][b, 4 * h:4 * h + 4].double().cpu().numpy(), w, to, f"{b} {h}")


def test_on_another_stream_and_in_a_graph(ta, dev, step):
    """The same bits on a stream of its own, and from every replay of a captured
    graph with other work in between."""
    x, bufs, _, _ = step
    f = x["f"]

    def state():
        return _clone(ta, f), f.sl.clone(), bufs()

    (c, t), sl, out = state()
    _step(ta, **x, cache=c, tail=t, sl=sl, bufs=out)
    torch.cuda.synchronize()

    def same(c2, t2, sl2, out2):
        torch.cuda.synchronize()
        _same_state(c, t, c2, t2)
        assert torch.equal(sl, sl2)
        for a, b in zip(out[:6], out2[:6]):
            assert torch.equal(a, b)

    (c2, t2), sl2, out2 = state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(ta, **x, cache=c2, tail=t2, sl=sl2, bufs=out2)
    same(c2, t2, sl2, out2)

    (c3, t3), sl3, out3 = state()
    first = [y.clone() for y in (c3.pages, c3.group_meta, c3.group_scale, t3.k, t3.v, sl3)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(ta, **x, cache=c3, tail=t3, sl=sl3, bufs=out3)
    for _ in range(3):
        for y, z in zip((c3.pages, c3.group_meta, c3.group_scale, t3.k, t3.v, sl3), first):
            y.copy_(z)
        for y in out3[:6]:
            y.zero_()
        graph.replay()
        same(c3, t3, sl3, out3)
        torch.randn(1 << 20, device=dev).sum().item()  # the program's own work
