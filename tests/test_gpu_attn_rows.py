"""turbo_attn_tree and turbo_attn_selected against 64 bits (tests/serving_ref.py
derives the bounds), over head layouts, lengths, masks and tables where they can go
wrong."""
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


def _words(see, dev):
    return torch.from_numpy(ref.matrix_to_words(see)).to(dev)


def _trees(kind, B, T, lens, seed):
    """(see, given as words or None) of one of the mask kinds."""
    rng = np.random.default_rng(seed)
    if kind == "chain":
        return np.tril(np.ones((T, T), bool))[None].repeat(B, 0)
    if kind == "tree":
        parents = np.stack([[rng.integers(-1, i) if i else -1 for i in range(T)] for _ in range(B)])
        return ref.ancestors(parents, [T] * B)[0]
    see = rng.random((B, T, T)) < 0.3  # any bits, rows that see no node among them
    see[:, ::3] = False
    return see


def _check(got, want, tol, what):
    err = np.abs(got - want)
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {err[bad].max()} over {tol[bad].min()} at {np.argwhere(bad)[0]}"


def _check_tree(f, q, kt, vt, see, tl, o, lse, o0=None, lse0=None, sm=ref.SM):
    B, Hq, T, _ = q.shape
    G = Hq // f.Hkv
    f.host()
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    for b in range(B):
        t = min(max(tl[b], 0), T)
        for h in range(f.Hkv):
            k, v = f.kv(b, h, range(f.groups(b)))
            n = len(k)
            k = np.concatenate([k, kt[b, h, :t].double().numpy()])
            v = np.concatenate([v, vt[b, h, :t].double().numpy()])
            vis = np.concatenate([np.ones((t, n), bool), see[b, :t, :t]], 1)
            for r in range(h * G, h * G + G):
                w, wl, to, tol = ref.attend(q[b, r, :t].double().numpy(), k, v, vis, sm)
                _check(o[b, r, :t], w, to, f"o of sequence {b}, head {r}")
                none = np.isneginf(wl)
                assert (np.isneginf(lse[b, r, :t]) == none).all()
                _check(lse[b, r, :t][~none], wl[~none], tol[~none], f"lse of sequence {b}, head {r}")
        if o0 is not None:  # rows behind the tree's last node
            assert (o[b, :, t:] == o0[b, :, t:].double().cpu().numpy()).all()
            assert (lse[b, :, t:] == lse0[b, :, t:].double().cpu().numpy()).all()


# B, Hq, Hkv, bits of the KV heads, lengths, T, tree lengths, mask, buffer
TREES = [
    (1, 1, 1, [4], [64], 1, [1], "tree", True),
    (1, 4, 4, [4, 2, 4, 2], [0], 5, [5], "any", True),          # no token, some rows empty
    (2, 4, 2, [2, 4], [0, 63], 7, [7, 3], "any", False),        # neither cache nor buffer
    (2, 2, 1, [2], [63, 65], 16, [16, 0], "chain", True),
    (3, 8, 2, [4, 2], [1, 64, 64 * 5 + 17], 17, [17, 1, 9], "tree", True),
    (2, 32, 2, [2, 4], [64 * 9 + 63, 64 * 33], 3, [3, 2], "tree", True),     # 16 heads a KV head
    (1, 10, 2, [4, 2], [64 * 40 + 5], 63, [63], "any", True),                # 5 heads a KV head
    (2, 6, 2, [4, 4], [64 * 70, 64 * 3], 64, [64, 50], "tree", False),
    (2, 4, 2, [2, 4], [64 * 12 + 1, 30], 65, [65, 64], "any", True),
    (1, 8, 1, [4], [64 * 21 + 40], 129, [129], "chain", True),
    (2, 4, 4, [4, 2, 2, 4], [64 * 4 + 9, 64 * 130], 256, [256, 200], "tree", True),
    (1, 4, 1, [2], [64 * 140 + 9], 30, [30], "tree", True),     # past 64 table entries
    (1, 2, 1, [4], [64 * 66], 64, [64], "any", False),
    (2, 16, 1, [4], [64 * 4 + 2, 64 * 17], 8, [8, 5], "tree", True),
    (2, 12, 2, [4, 2], [64 * 9 + 5, 64 * 70 + 1], 100, [100, 37], "any", True),  # 600 rows
    (1, 16, 1, [2], [64 * 20 + 63], 64, [64], "tree", False),
    (9, 8, 8, [4, 2] * 4, [64 * i + 7 * i for i in range(9)], 4, [4, 3, 2, 1, 0, 4, 4, 4, 4], "tree", True),
]


@pytest.mark.parametrize("case", range(len(TREES)))
def test_tree_against_64_bits(ta, dev, case):
    B, Hq, Hkv, bits, lens, T, tl, kind, tail = TREES[case]
    print("tree", TREES[case], flush=True)
    f = ref.Filled(ta, dev, lens, bits, seed=case + 1, tail=tail)
    q, kt, vt = ref.rand((B, Hq, T, D), 1), ref.rand((B, Hkv, T, D), 2), ref.rand((B, Hkv, T, D), 3)
    kt[..., 7] *= 10
    see = _trees(kind, B, T, tl, case)
    g = Guarded(dev)
    o, lse = g((B, Hq, T, D), torch.float16), g((B, Hq, T), torch.float32)
    n = ta.lib().turbo_tree_workspace_bytes(B, Hq, Hkv, T, f.mg, int(tail))
    ws = g((n // 4,), torch.float32) if n else None
    o.fill_(3.0)
    lse.fill_(4.0)
    o0, lse0 = o.clone(), lse.clone()
    args = (q.to(dev), kt.to(dev), vt.to(dev), None if kind == "chain" else _words(see, dev),
            torch.tensor(tl, dtype=torch.int32, device=dev), f.cache, f.sl, f.btd, f.gtd)
    ta.turbo_attn_tree(*args, tail=f.tail, workspace=ws, out=o, lse_out=lse)
    g.check("turbo_attn_tree")
    _check_tree(f, q, kt, vt, see, tl, o, lse, o0, lse0)
    again = ta.turbo_attn_tree(*args, tail=f.tail, out=o0, lse_out=lse0)
    assert torch.equal(again[0].view(torch.int16), o.view(torch.int16))
    assert torch.equal(again[1].view(torch.int32), lse.view(torch.int32))


@pytest.mark.parametrize("scale,sm", [(1.0, 1.0), (12.0, ref.SM), (2.0 ** -12, ref.SM), (0.02, 30.0)])
def test_tree_ranges(ta, dev, scale, sm):
    """Scores far apart (one token takes all), and queries in fp16's subnormals."""
    B, Hq, Hkv, T = 1, 4, 2, 12
    f = ref.Filled(ta, dev, [64 * 6 + 30], [4, 2], seed=31)
    q, kt, vt = ref.rand((B, Hq, T, D), 1, scale), ref.rand((B, Hkv, T, D), 2), ref.rand((B, Hkv, T, D), 3)
    see = _trees("tree", B, T, [T], 3)
    o, lse = ta.turbo_attn_tree(q.to(dev), kt.to(dev), vt.to(dev), _words(see, dev),
                                torch.tensor([T], dtype=torch.int32, device=dev), f.cache, f.sl,
                                f.btd, f.gtd, sm_scale=sm, tail=f.tail, return_lse=True)
    _check_tree(f, q, kt, vt, see, [T], o, lse, sm=sm)


@pytest.mark.parametrize("Hq,T,tl", [(4, 70, [66, 40]), (2, 40, [40, 35]), (2, 16, [16, 9])])
def test_tree_rows_do_not_see_what_their_mask_hides(ta, dev, Hq, T, tl):
    """Infinities and NaN in nodes a row does not see, and behind the tree's last,
    change nothing; in nodes it sees they do what the formula does."""
    B, Hkv = 2, 2
    f = ref.Filled(ta, dev, [64 * 3 + 20, 64 * 8], [4, 2], seed=41)
    q, kt, vt = ref.rand((B, Hq, T, D), 1), ref.rand((B, Hkv, T, D), 2), ref.rand((B, Hkv, T, D), 3)
    see = _trees("tree", B, T, tl, 5)
    hidden = [i for i in (0, 3, 8, 17, 33, 64) if i < T]
    see[:, :, hidden] = False
    clean = [x.clone() for x in (kt, vt)]
    bad = [float("nan"), float("inf"), float("-inf")]
    for i, h in enumerate(hidden):
        kt[:, :, h], vt[:, :, h] = bad[i % 3], bad[(i + 1) % 3]
    for b in range(B):
        kt[b, :, tl[b]:] = float("nan")
        vt[b, :, tl[b]:] = float("inf")
    tld = torch.tensor(tl, dtype=torch.int32, device=dev)

    def run(k, v, m):
        o, lse = (torch.zeros(B, Hq, T, D, dtype=torch.float16, device=dev),
                  torch.zeros(B, Hq, T, device=dev))
        ta.turbo_attn_tree(q.to(dev), k.to(dev), v.to(dev), _words(m, dev), tld, f.cache, f.sl,
                           f.btd, f.gtd, tail=f.tail, out=o, lse_out=lse)
        return o, lse

    a, b_ = run(kt, vt, see), run(*clean, see)
    assert torch.equal(a[0].view(torch.int16), b_[0].view(torch.int16)) and torch.equal(a[1], b_[1])
    # node 2 sees an infinite value, node 5 one that is not a number, node 6 such a key
    for far in (h for h in hidden if h < min(tl)):
        seen = see.copy()
        seen[:, 2, far], seen[:, 5, far], seen[:, 6, far] = True, True, True
        for which, row, value in (("v", 2, float("inf")), ("v", 5, float("nan")), ("k", 6, float("nan"))):
            k2, v2 = clean[0].clone(), clean[1].clone()
            (v2 if which == "v" else k2)[:, :, far, 5] = value
            o, lse = run(k2, v2, seen)
            cut = [i for i in range(T) if i not in (2, 5, 6)]
            assert torch.equal(o[:, :, cut].view(torch.int16), b_[0][:, :, cut].view(torch.int16))
            if which == "k":
                assert torch.isnan(o[:, :, row]).all() and torch.isnan(lse[:, :, row]).all()
            else:
                x = o[:, :, row, 5]
                assert (torch.isnan(x) if value != value else torch.isinf(x)).all()
                assert torch.isfinite(o[:, :, row, 6:]).all() and torch.isfinite(o[:, :, row, :5]).all()


def test_tree_large_finite_values(ta, dev):
    """Values at fp16's ends in visible nodes: sums stay in binary32's range."""
    f = ref.Filled(ta, dev, [64 * 2], [4], seed=51)
    T = 9
    q, kt, vt = ref.rand((1, 1, T, D), 1), ref.rand((1, 1, T, D), 2), ref.rand((1, 1, T, D), 3)
    vt[0, 0, ::2] = 65504.0
    vt[0, 0, 1::2] = -65504.0
    see = _trees("any", 1, T, [T], 1)
    o, lse = ta.turbo_attn_tree(q.to(dev), kt.to(dev), vt.to(dev), _words(see, dev),
                                torch.tensor([T], dtype=torch.int32, device=dev), f.cache, f.sl,
                                f.btd, f.gtd, tail=f.tail, return_lse=True)
    _check_tree(f, q, kt, vt, see, [T], o, lse)


def test_tree_skips_groups_outside_the_tables_ranges(ta, dev):
    """Groups with an entry out of range are not read; max_groups cuts the cache."""
    B, Hq, Hkv, T = 2, 4, 2, 6
    f = ref.Filled(ta, dev, [64 * 9 + 11, 64 * 9], [4, 2], seed=61)
    f.bt[0, 4 * 2 + 1], f.bt[0, 4 * 5] = -1, f.cache.pages.shape[0]
    f.gt[0, 7], f.gt[1, 0], f.gt[1, 8] = -5, f.cache.group_meta.shape[0], 2 ** 31 - 1
    f.btd.copy_(torch.from_numpy(f.bt))
    f.gtd.copy_(torch.from_numpy(f.gt))
    q, kt, vt = ref.rand((B, Hq, T, D), 1), ref.rand((B, Hkv, T, D), 2), ref.rand((B, Hkv, T, D), 3)
    see = _trees("tree", B, T, [T] * B, 3)
    o, lse = ta.turbo_attn_tree(q.to(dev), kt.to(dev), vt.to(dev), _words(see, dev),
                                torch.tensor([T, T], dtype=torch.int32, device=dev), f.cache, f.sl,
                                f.btd, f.gtd, tail=f.tail, return_lse=True)
    _check_tree(f, q, kt, vt, see, [T] * B, o, lse)
    # lengths past the tables: the full groups they hold (no buffer: none is addressed)
    f.sl.fill_(64 * 40 + 3)
    f.lens, f.tail = [64 * 40 + 3] * 2, None
    o, lse = ta.turbo_attn_tree(q.to(dev), kt.to(dev), vt.to(dev), _words(see, dev),
                                torch.tensor([T, 99], dtype=torch.int32, device=dev), f.cache, f.sl,
                                f.btd, f.gtd, return_lse=True)
    _check_tree(f, q, kt, vt, see, [T, 99], o, lse)
    # a negative length: nothing cached
    f.sl.fill_(-3)
    f.lens = [-3] * 2
    o, lse = ta.turbo_attn_tree(q.to(dev), kt.to(dev), vt.to(dev), _words(see, dev),
                                torch.tensor([T, T], dtype=torch.int32, device=dev), f.cache, f.sl,
                                f.btd, f.gtd, return_lse=True)
    _check_tree(f, q, kt, vt, see, [T] * B, o, lse)


@pytest.mark.parametrize("Hq,T", [(2, 3), (4, 24), (4, 90)])
def test_scales_of_zero_and_far_apart(ta, dev, Hq, T):
    """Groups and buffers whose scales are zero, subnormal or far from the others'."""
    B, Hkv = 2, 2
    f = ref.Filled(ta, dev, [64 * 14 + 20, 64 * 3 + 5], [4, 2], seed=65)
    sc = f.cache.group_scale
    for i, (sk, sv) in enumerate([(None, 0.0), (0.0, None), (None, 1e-42), (1e-42, None), (None, 1e-30),
                                  (None, 50.0), (0.0, 0.0), (None, 1e-4)]):
        slot = f.gtd[0, i].long()
        if sk is not None:
            sc[slot, :, 0] = sk
        if sv is not None:
            sc[slot, :, 1] = sv
    sc[f.gtd[1].long()[:3], :, 1] = torch.tensor([0.0, 1e-42, 0.0], device=dev)[:, None]
    f.tail.scale[0, 0], f.tail.scale[1, 0], f.tail.scale[1, 1, 1] = 0.0, 1e-42, 0.0
    q, kt, vt = ref.rand((B, Hq, T, D), 1), ref.rand((B, Hkv, T, D), 2), ref.rand((B, Hkv, T, D), 3)
    see = _trees("any", B, T, [T] * B, 3)
    o, lse = ta.turbo_attn_tree(q.to(dev), kt.to(dev), vt.to(dev), _words(see, dev),
                                torch.tensor([T, T], dtype=torch.int32, device=dev), f.cache, f.sl,
                                f.btd, f.gtd, tail=f.tail, return_lse=True)
    _check_tree(f, q, kt, vt, see, [T] * B, o, lse)
    # no number in the scale of one group: none in the rows that attend it
    sc[f.gtd[0, 9].long(), 1, 1] = float("nan")
    o2, lse2 = ta.turbo_attn_tree(q.to(dev), kt.to(dev), vt.to(dev), _words(see, dev),
                                  torch.tensor([T, T], dtype=torch.int32, device=dev), f.cache, f.sl,
                                  f.btd, f.gtd, tail=f.tail, return_lse=True)
    G = Hq // Hkv
    assert torch.isnan(o2[0, G:]).all() and torch.equal(o2[0, :G], o[0, :G]) and torch.equal(o2[1], o[1])


def test_operands_at_any_fp16_boundary(ta, dev):
    B, Hq, Hkv, T = 1, 4, 2, 20
    f = ref.Filled(ta, dev, [64 * 4 + 10], [4, 2], seed=71)
    q, kt, vt = ref.rand((B, Hq, T, D), 1), ref.rand((B, Hkv, T, D), 2), ref.rand((B, Hkv, T, D), 3)
    see = _trees("tree", B, T, [T], 3)
    tl = torch.tensor([T], dtype=torch.int32, device=dev)

    def odd(x, at):
        buf = torch.zeros(x.numel() + 8, dtype=torch.float16, device=dev)
        v = buf[at:at + x.numel()].view(x.shape)
        return v.copy_(x)

    want = ta.turbo_attn_tree(q.to(dev), kt.to(dev), vt.to(dev), _words(see, dev), tl, f.cache, f.sl,
                              f.btd, f.gtd, tail=f.tail, return_lse=True)
    out = odd(torch.zeros_like(q), 5)
    got = ta.turbo_attn_tree(odd(q, 1), odd(kt, 3), odd(vt, 7), _words(see, dev), tl, f.cache, f.sl,
                             f.btd, f.gtd, tail=f.tail, return_lse=True, out=out)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    sel = torch.arange(4, dtype=torch.int32, device=dev).expand(1, Hkv, 4).contiguous()
    q1 = q[:, :, 0].contiguous()
    want = ta.turbo_attn_selected(q1.to(dev), f.cache, f.sl, f.btd, f.gtd, sel, tail=f.tail)
    got = ta.turbo_attn_selected(odd(q1, 1), f.cache, f.sl, f.btd, f.gtd, sel, tail=f.tail,
                                 out=odd(torch.zeros_like(q1), 3))
    assert torch.equal(got, want)


# Hq, bits, lengths, num_select, buffer
CHOICES = [
    (1, [4], [64 * 3], 1, False),
    (4, [4, 2], [64 * 5 + 9, 63, 0], 3, True),
    (16, [2], [64 * 30 + 1, 64], 40, True),      # more entries than groups
    (10, [4, 2], [64 * 90 + 63], 17, False),
    (6, [2, 4, 4], [64 * 11, 64 * 20 + 5], 8, True),
    (40, [4, 2] * 5, [64 * 128 + 30] * 3, 100, True),
]


@pytest.mark.parametrize("case", range(len(CHOICES)))
def test_selected_against_64_bits(ta, dev, case):
    Hq, bits, lens, k, tail = CHOICES[case]
    print("selected", CHOICES[case], flush=True)
    B, Hkv = len(lens), len(bits)
    G = Hq // Hkv
    f = ref.Filled(ta, dev, lens, bits, seed=case + 81, tail=tail)
    rng = np.random.default_rng(case)
    sel = np.full((B, Hkv, k), -1, np.int32)  # in any order, some past the sequence's groups
    for b in range(B):
        for h in range(Hkv):
            x = rng.permutation(f.groups(b) + 2)[:k]
            sel[b, h, :len(x)] = x
    if k > 2:  # the same group twice, and entries that are no group
        sel[:, 0, 1] = sel[:, 0, 0]
        sel[:, -1, 2] = 2 ** 31 - 1
    q = ref.rand((B, Hq, D), 1)
    g = Guarded(dev)
    o, lse = g((B, Hq, D), torch.float16), g((B, Hq), torch.float32)
    n = ta.lib().turbo_selected_workspace_bytes(B, Hq, Hkv, k, int(tail))
    ws = g((n // 4,), torch.float32) if n else None
    seld = torch.from_numpy(sel).to(dev)
    ta.turbo_attn_selected(q.to(dev), f.cache, f.sl, f.btd, f.gtd, seld, workspace=ws, out=o,
                           lse_out=lse, tail=f.tail)
    g.check("turbo_attn_selected")
    f.host()
    for b in range(B):
        for h in range(Hkv):
            kk, vv = f.kv(b, h, [x for x in sel[b, h] if 0 <= x < f.groups(b)])
            w, wl, to, tol = ref.attend(q[b, h * G:h * G + G].double().numpy(), kk, vv)
            _check(o[b, h * G:h * G + G].double().cpu().numpy(), w, to, f"o {b} {h}")
            got = lse[b, h * G:h * G + G].double().cpu().numpy()
            assert (np.isneginf(got) == np.isneginf(wl)).all()
            if len(kk):
                _check(got, wl, tol, f"lse {b} {h}")


def test_selected_every_group_is_near_the_decode(ta, dev):
    """Every group chosen: the attention that turbo_attn_decode approximates with
    SAS, int8 queries and probabilities (its outputs within a few per cent)."""
    lens, bits, Hq = [64 * 20 + 31, 64 * 7], [4, 2], 8
    f = ref.Filled(ta, dev, lens, bits, seed=95)
    q = ref.rand((2, Hq, D), 5).to(dev)
    sel = torch.arange(f.mg, dtype=torch.int32, device=dev).expand(2, 2, f.mg).contiguous()
    o, lse = ta.turbo_attn_selected(q, f.cache, f.sl, f.btd, f.gtd, sel, tail=f.tail, return_lse=True)
    d, dl = ta.turbo_attn_decode(q, f.cache, f.sl, f.btd, f.gtd, tail=f.tail, return_lse=True)
    assert ((o - d).float().norm() / d.float().norm()).item() < 0.1
    assert (lse - dl).abs().max().item() < 0.1


@pytest.mark.parametrize("B,T", [(32, 66), (33, 20), (8, 260 // 2), (4, 3)])
def test_long_sequences_in_a_batch(ta, dev, B, T):
    """Chunks of more tiles than one round of table entries: B sequences that are the
    same one of 18000 tokens, four of its rows against 64 bits, all alike."""
    Hkv, Hq, bits = 4, 8 if T == 130 else 4, [4, 2, 2, 4]
    f = ref.Filled(ta, dev, [18000], bits, seed=97)
    q, kt, vt = ref.rand((1, Hq, T, D), 1), ref.rand((1, Hkv, T, D), 2), ref.rand((1, Hkv, T, D), 3)
    see = _trees("tree", 1, T, [T], 3)
    tail = ta.KVTail(B, Hkv, dev)
    for x, y in ((tail.k, f.tail.k), (tail.v, f.tail.v), (tail.scale, f.tail.scale)):
        x.copy_(y.expand(x.shape))

    def all_of(x):
        return x.to(dev).expand(B, *x.shape[1:]).contiguous()

    o, lse = ta.turbo_attn_tree(all_of(q), all_of(kt), all_of(vt), all_of(_words(see, dev)),
                                torch.full((B,), T, dtype=torch.int32, device=dev), f.cache,
                                all_of(f.sl[None])[:, 0].contiguous(), all_of(f.btd), all_of(f.gtd),
                                tail=tail, return_lse=True)
    assert torch.equal(o, o[:1].expand_as(o)) and torch.equal(lse, lse[:1].expand_as(lse))
    f.host()
    for h in range(Hkv):
        k, v = f.kv(0, h, range(f.groups(0)))
        k, v = np.concatenate([k, kt[0, h].double().numpy()]), np.concatenate([v, vt[0, h].double().numpy()])
        r, i = h * (Hq // Hkv), [0, T // 2, T - 1]
        vis = np.concatenate([np.ones((T, len(k) - T), bool), see[0]], 1)[i]
        w, wl, to, tol = ref.attend(q[0, r, i].double().numpy(), k, v, vis)
        _check(o[0, r, i].double().cpu().numpy(), w, to, f"o {h}")
        _check(lse[0, r, i].double().cpu().numpy(), wl, tol, f"lse {h}")


@pytest.mark.parametrize("B,Hkv,T,ng", [(64, 4, 1, 5200), (1, 2, 40, 700), (8, 4, 70, 5000)])
def test_very_long_tables(ta, dev, B, Hkv, T, ng):
    """Sequences of up to 333000 tokens (three groups of keys and values over and over),
    beside short ones in tables as wide: every round of table entries, every chunk."""
    bits = [4, 2] * (Hkv // 2)
    f = ref.Filled(ta, dev, [64 * 3], bits, seed=99, tail=False)
    kind = np.random.default_rng(ng).integers(0, 3, ng)
    count = np.bincount(kind, minlength=3)
    gt = np.repeat(f.gt[0][kind][None], B, 0).astype(np.int32)
    bt = np.repeat(f.bt[0].reshape(-1, 4)[kind].reshape(1, -1), B, 0).astype(np.int32)
    lens = [64 * ng if b % 3 == 0 else 64 * (b % 7) for b in range(B)]
    q, kt, vt = (ref.rand((1, Hkv, T, D), i).expand(B, -1, -1, -1).contiguous() for i in (1, 2, 3))
    i32 = dict(dtype=torch.int32, device=dev)
    o, lse = ta.turbo_attn_tree(q.to(dev), kt.to(dev), vt.to(dev), None, torch.full((B,), T, **i32),
                                f.cache, torch.tensor(lens, **i32), torch.from_numpy(bt).to(dev),
                                torch.from_numpy(gt).to(dev), return_lse=True)
    f.host()
    for b in sorted({0, 1 % B, 2 % B, B - 1}):
        n = lens[b] // 64
        c = np.bincount(kind[:n], minlength=3)
        for h in range(Hkv):
            k, v = f.kv(0, h, range(3))
            for i in sorted({0, T // 2, T - 1}):
                # a token seen c times weighs c times: its score plus ln c
                kk = np.concatenate([k, kt[b, h, :i + 1].double().numpy()])
                vv = np.concatenate([v, vt[b, h, :i + 1].double().numpy()])
                w = np.concatenate([np.repeat(c, 64), np.ones(i + 1)])
                x = ref.SM * (kk @ q[b, h, i].double().numpy())
                p = np.exp(x - x.max()) * w
                want, l = p @ vv / p.sum(), x.max() + np.log(p.sum())
                _, _, to, tol = ref.attend(q[b, h, i:i + 1].double().numpy(), kk, vv)
                # (n tokens instead of a few hundred in the row's sums)
                more = (w.sum() / 16) * 2.0 ** -24
                a = p @ np.abs(vv) / p.sum()
                to = ref.F16 * np.abs(want) + 2.0 ** -25 + a * (ref.F16 + more + 2.0 ** -19)
                _check(o[b, h, i].double().cpu().numpy(), want, to, f"o {b} {h} {i}")
                assert abs(lse[b, h, i].item() - l) <= tol[0] + more + 2.0 ** -22 * abs(l)


def test_long_cache_past_32_bit_offsets(ta, dev):
    """Pages beyond 4 GiB of the pool."""
    bits = [4] * 64
    pb = ta.page_bytes(bits)  # 128 KiB
    npages = (5 << 30) // pb
    c = ta.PagedKVCache(1, 2, bits, dev)
    c.pages = torch.empty(npages, pb, dtype=torch.uint8, device=dev)
    k, v = ref.rand((1, 64, 128, D), 1), ref.rand((1, 64, 128, D), 2)
    bt = torch.tensor([[npages - 1, 3, npages - 2, 9, 0, npages - 7, 1, npages - 5]], dtype=torch.int32, device=dev)
    gt = torch.tensor([[1, 0]], dtype=torch.int32, device=dev)
    ta.turbo_quantize_kv(k.to(dev), v.to(dev), c, bt, gt)
    small = ta.PagedKVCache(8, 2, bits, dev)
    bs = torch.arange(8, dtype=torch.int32, device=dev).view(1, 8)
    ta.turbo_quantize_kv(k.to(dev), v.to(dev), small, bs, gt)
    sl = torch.tensor([128], dtype=torch.int32, device=dev)
    q = ref.rand((1, 64, 3, D), 3).to(dev)
    kt, vt = ref.rand((1, 64, 3, D), 4).to(dev), ref.rand((1, 64, 3, D), 5).to(dev)
    tl = torch.tensor([3], dtype=torch.int32, device=dev)
    a = ta.turbo_attn_tree(q, kt, vt, None, tl, c, sl, bt, gt)
    b = ta.turbo_attn_tree(q, kt, vt, None, tl, small, sl, bs, gt)
    assert torch.equal(a, b) and torch.isfinite(a).all()
