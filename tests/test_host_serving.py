"""Refusals and sizes of the sparse and speculative decoding calls (no GPU)."""
import ctypes

import pytest
import torch

import paper_2412_08585_amd as ta
from paper_2412_08585_amd import binding

P = ctypes.c_void_p
DUMMY = P(256)


def _cache(bits=(4, 4)):
    c = ta.TurboKVCacheStruct()
    c.pages, c.group_meta, c.group_scale = 256, 256, 256
    c.num_pages, c.num_group_slots, c.num_kv_heads, c.head_dim = 8, 2, len(bits), 128
    for i, b in enumerate(bits):
        c.head_bits[i] = b
    return c


def _tail(batch=1, heads=2, **kw):
    t = ta.TurboKVTailStruct()
    t.k, t.v, t.scale, t.batch, t.num_kv_heads = 256, 256, 256, batch, heads
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def _ref(x):
    return None if x is None else ctypes.byref(x)


@pytest.fixture(scope="module")
def L():
    return ta.lib()


def _select(L, c=None, B=1, Hq=4, mg=2, num=2, first=1, last=1, ws=DUMMY, n=1 << 20, sel=DUMMY,
            q=DUMMY):
    return L.turbo_select_groups(q, _ref(_cache() if c is None else c), DUMMY, DUMMY, DUMMY, mg, B,
                                 Hq, num, first, last, ws, n, sel, None)


def _selected(L, c=None, tail=None, B=1, Hq=4, mg=2, num=2, sm=0.1, ws=DUMMY, n=1 << 20, o=DUMMY,
              sel=DUMMY):
    return L.turbo_attn_selected(DUMMY, _ref(_cache() if c is None else c), _ref(tail), DUMMY, DUMMY,
                                 DUMMY, mg, sel, num, B, Hq, sm, ws, n, o, None, None)


def _tree(L, c=None, tail=None, B=1, Hq=4, T=4, mg=2, sm=0.1, ws=DUMMY, n=1 << 20, o=DUMMY,
          kt=DUMMY, lens=DUMMY):
    return L.turbo_attn_tree(DUMMY, kt, DUMMY, DUMMY, lens, _ref(_cache() if c is None else c),
                             _ref(tail), DUMMY, DUMMY, DUMMY, mg, B, Hq, T, sm, ws, n, o, None, None)


def _path(L, c=None, tail=None, B=1, Hkv=2, T=4, d=128, P_=3, mg=2, path=DUMMY):
    return L.turbo_append_path(DUMMY, DUMMY, B, Hkv, T, d, path, DUMMY, P_, DUMMY,
                               _ref(_cache() if c is None else c), _ref(_tail() if tail is None else tail),
                               DUMMY, DUMMY, mg, None)


NAN = float("nan")


def test_refused_before_any_launch(L):
    for call in (_select, _selected, _tree):
        assert call(L, B=-1) == -1 and call(L, Hq=0) == -1 and call(L, mg=0) == -1
        assert call(L, Hq=5) == -1 and call(L, Hq=34) == -1  # not a multiple; 17 rows a KV head
        assert call(L, c=_cache((4, 3))) == -1
        assert call(L, B=0) == 0
        bad = _cache()
        bad.head_dim = 64
        assert call(L, c=bad) == -1
        bad = _cache()
        bad.pages = None
        assert call(L, c=bad) == -1
    for call in (_selected, _tree):
        for sm in (0.0, -1.0, NAN, float("inf")):
            assert call(L, sm=sm) == -1
        assert call(L, o=None) == -1
        assert call(L, tail=_tail(heads=1)) == -1 and call(L, tail=_tail(k=None)) == -1
        assert call(L, B=2, tail=_tail(batch=1)) == -1
    for kw in (dict(num=0), dict(first=-1), dict(last=-1), dict(first=2, last=1), dict(first=3, last=0),
               dict(first=2 ** 31 - 1, last=2 ** 31 - 1), dict(sel=None), dict(q=None)):
        assert _select(L, **kw) == -1, kw
    assert _select(L, ws=None) == -3 and _select(L, n=4 * 4 * 2 - 1) == -3
    assert _select(L, B=2 ** 24, mg=64 * 256) == -1  # more work-groups than a launch has
    assert _selected(L, num=0) == -1 and _selected(L, sel=None) == -1
    for T in (0, -1, 257):
        assert _tree(L, T=T) == -1 and _path(L, T=T) == -1
        assert L.turbo_tree_mask(DUMMY, DUMMY, 1, T, DUMMY, None, None) == -1
    assert _tree(L, kt=None) == -1 and _tree(L, lens=None) == -1
    assert _tree(L, B=2 ** 21, T=256, n=1 << 62) == -1  # more rows than an index has
    assert L.turbo_tree_mask(None, DUMMY, 1, 4, DUMMY, None, None) == -1
    assert L.turbo_tree_mask(DUMMY, DUMMY, -1, 4, DUMMY, None, None) == -1
    assert L.turbo_tree_mask(None, None, 0, 4, None, None, None) == 0
    for kw in (dict(B=-1), dict(Hkv=0), dict(Hkv=65), dict(Hkv=3), dict(d=64), dict(P_=0), dict(mg=0),
               dict(path=None), dict(tail=_tail(heads=1)), dict(B=2), dict(c=_cache((4, 5)))):
        assert _path(L, **kw) == -1, kw
    assert _path(L, B=0) == 0


def test_workspace_sizes(L):
    assert L.turbo_select_workspace_bytes(3, 8, 5) == 3 * 8 * 5 * 4
    for args in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (-1, 1, 1)):
        assert L.turbo_select_workspace_bytes(*args) == 0
    for args in ((0, 4, 2, 8, 1), (1, 0, 2, 8, 1), (1, 4, 0, 8, 1), (1, 5, 2, 8, 1), (1, 4, 2, 0, 1)):
        assert L.turbo_selected_workspace_bytes(*args) == 0
    for args in ((0, 4, 2, 8, 9, 1), (1, 5, 2, 8, 9, 1), (1, 4, 2, 0, 9, 1), (1, 4, 2, 257, 9, 1),
                 (1, 4, 2, 8, 0, 1)):
        assert L.turbo_tree_workspace_bytes(*args) == 0
    # a long cache of one sequence is cut into chunks, whose states are 132 words a row
    for n in (L.turbo_selected_workspace_bytes(1, 32, 8, 64, 1) / 32,
              L.turbo_tree_workspace_bytes(1, 32, 8, 16, 512, 1) / (32 * 16)):
        assert n >= 2 * 528 and n % 528 == 0
    # and refused without them
    c = _cache((4,) * 8)
    assert _selected(L, c=c, Hq=32, num=64, mg=512, ws=None) == -3
    need = L.turbo_tree_workspace_bytes(1, 32, 8, 16, 512, 0)
    assert _tree(L, c=c, Hq=32, T=16, mg=512, n=need - 1) == -3


def test_the_binding_names_what_is_wrong():
    """Types, shapes, devices and orders are checked before the library is called."""
    B, Hq, Hkv, T, mg = 2, 4, 2, 5, 3
    c, t = ta.PagedKVCache(4, 2, [4, 2], "cpu"), ta.KVTail(B, Hkv, "cpu")
    f16, i32 = torch.float16, torch.int32
    q = torch.zeros(B, Hq, 128, dtype=f16)
    sl, bt, gt = torch.zeros(B, dtype=i32), torch.zeros(B, 4 * mg, dtype=i32), torch.zeros(B, mg, dtype=i32)
    sel = torch.zeros(B, Hkv, 2, dtype=i32)
    ok = (q, c, sl, bt, gt)

    def swap(args, i, x):
        return args[:i] + (x,) + args[i + 1:]

    for args, what in ((swap(ok, 0, q.float()), "q must"), (swap(ok, 0, q[0]), "q must"),
                       (swap(ok, 0, torch.zeros(B, Hq, 64, dtype=f16)), "q must"),
                       (swap(ok, 0, torch.zeros(B, 128, Hq, dtype=f16).transpose(1, 2)), "contiguous"),
                       (swap(ok, 2, sl.long()), "seq_lens"), (swap(ok, 2, sl[:1]), "seq_lens"),
                       (swap(ok, 3, bt[:, :-1]), "block_table"), (swap(ok, 4, gt[0]), "group_table")):
        with pytest.raises(ValueError, match=what):
            ta.turbo_select_groups(*args, 2)
        with pytest.raises(ValueError, match=what):
            ta.turbo_attn_selected(*args, sel)
    for n in (0, -1):
        with pytest.raises(ValueError, match="num_select"):
            ta.turbo_select_groups(*ok, n)
    with pytest.raises(ValueError, match="selected"):
        ta.turbo_attn_selected(*ok, sel[:, :1])
    with pytest.raises(ValueError, match="out must"):
        ta.turbo_attn_selected(*ok, sel, out=q.float())
    with pytest.raises(ValueError, match="lse_out"):
        ta.turbo_attn_selected(*ok, sel, lse_out=torch.zeros(B, Hq, 1))
    with pytest.raises(ValueError, match="cuda"):  # all is well but the device
        ta.turbo_attn_selected(*ok, sel, workspace=torch.zeros(1 << 16))
    qt = torch.zeros(B, Hq, T, 128, dtype=f16)
    kt = torch.zeros(B, Hkv, T, 128, dtype=f16)
    m, tl = torch.zeros(B, T, 1, dtype=torch.int64), torch.zeros(B, dtype=i32)
    ok = (qt, kt, kt, m, tl, c, sl, bt, gt)
    for args, what in ((swap(ok, 0, q), "q must"), (swap(ok, 1, kt[:, :1]), "k_tree"),
                       (swap(ok, 2, kt.float()), "v_tree"), (swap(ok, 3, m.int()), "tree_mask"),
                       (swap(ok, 3, torch.zeros(B, T, 2, dtype=torch.int64)), "tree_mask"),
                       (swap(ok, 4, tl[:1]), "tree_lens")):
        with pytest.raises(ValueError, match=what):
            ta.turbo_attn_tree(*args)
    with pytest.raises(ValueError, match="parents"):
        ta.turbo_tree_mask(tl, tl)
    with pytest.raises(ValueError, match="tree_lens"):
        ta.turbo_tree_mask(torch.zeros(B, T, dtype=i32), tl[:1])
    path = torch.zeros(B, 3, dtype=i32)
    with pytest.raises(ValueError, match="path must"):
        ta.turbo_append_path(kt, kt, path.long(), tl, sl, c, t, bt, gt)
    with pytest.raises(ValueError, match="path_lens"):
        ta.turbo_append_path(kt, kt, path, path, sl, c, t, bt, gt)
    with pytest.raises(ValueError, match="v_tree"):
        ta.turbo_append_path(kt, kt[:, :, :2].contiguous(), path, tl, sl, c, t, bt, gt)


def test_every_call_is_public():
    for name in ("turbo_select_groups", "turbo_attn_selected", "turbo_tree_mask", "turbo_attn_tree",
                 "turbo_append_path", "select_workspace", "selected_workspace", "tree_workspace"):
        assert getattr(ta, name) is getattr(binding, name) and name in ta.__all__
