"""Speculative and sparse decoding over the compressed paged cache: the calls
whose speed is measured, with their plain forms.

Kinds of case (one pass each):
  select    choose the groups of the cache that a decoding step attends, from
            the bounds that the groups' scales and zero points give
  selected  one decoding step over such a choice and the int8 buffer
  mask      ancestor bits and depths of drafted trees, from parent indices
  tree      attention of drafted nodes over the cache, the buffer and the nodes
            they descend from
  path      append an accepted path of nodes to the buffer and the cache

Activations are N(0, 1), four key channels per (sequence, KV head) scaled by
10; page tables are shuffled; half of the KV heads have 2 bits in "mixed".
"""
import math
import random

import numpy as np
import torch

own = False

D = 128        # head dimension
GROUP = 64     # tokens of a cache group
PAGE = 16      # tokens of a page
QMAX = 119.0
FIRST, LAST = 1, 2  # groups that a selection always holds
HEADS = ((4, 4), (16, 16), (32, 16), (40, 10), (32, 8), (64, 8), (32, 2))
MAX_BYTES = 1.2e9   # minimal traffic of a drawn case, at most
MAX_FLOPS = 1.3e11
MAX_CACHE = 64 * 10 * 8192  # tokens times KV heads of a drawn cache, at most


def listed():
    return [
        # one long conversation: 512 groups to choose from
        dict(name="select-1x32k", kind="select", B=1, Hq=32, Hkv=8, N=32767, bits="int4",
             ragged=False, k=64),
        # a serving batch of every length, eight query heads per KV head
        dict(name="select-32x16k", kind="select", B=32, Hq=64, Hkv=8, N=16383, bits="mixed",
             ragged=True, k=32),
        # the long conversation's attention: an eighth of its groups
        dict(name="selected-1x32k", kind="selected", B=1, Hq=32, Hkv=8, N=32767, bits="int4",
             ragged=False, k=64),
        # the Phi-3-medium decode batch from a quarter of its cache
        dict(name="selected-64x8k", kind="selected", B=64, Hq=40, Hkv=10, N=8190, bits="mixed",
             ragged=False, k=32),
        # one small tree
        dict(name="mask-1x16", kind="mask", B=1, T=16),
        # the trees of a large batch, some of them short
        dict(name="mask-256x200", kind="mask", B=256, T=200),
        # one conversation's drafted tree: latency
        dict(name="tree-1x4k", kind="tree", B=1, Hq=32, Hkv=8, N=4000, bits="int4",
             ragged=False, T=16, chain=False),
        # the Phi-3-medium decode batch with a short drafted chain per sequence
        dict(name="tree-64x8k", kind="tree", B=64, Hq=40, Hkv=10, N=8190, bits="mixed",
             ragged=False, T=5, chain=True),
        # a ragged batch with trees of up to 63 nodes
        dict(name="tree-16x16k", kind="tree", B=16, Hq=64, Hkv=8, N=16383, bits="mixed",
             ragged=True, T=63, chain=False),
        # the widest tree over a long context: matrix products
        dict(name="tree-2x16k", kind="tree", B=2, Hq=32, Hkv=8, N=16384, bits="int4",
             ragged=False, T=256, chain=False),
        # one conversation's accepted nodes
        dict(name="path-1", kind="path", B=1, Hkv=8, N=4000, bits="int4", ragged=False, T=16, P=5),
        # a large batch's, some of which fill their buffer
        dict(name="path-256", kind="path", B=256, Hkv=10, N=1023, bits="mixed", ragged=True, T=64,
             P=16),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("select", "selected", "selected", "mask", "tree", "tree", "tree", "path"))
    if kind == "mask":
        return dict(kind=kind, B=_log_int(rng, 1, 256), T=_log_int(rng, 8, 256))
    while True:
        Hq, Hkv = rng.choice(HEADS)
        c = dict(kind=kind, B=_log_int(rng, 1, 256 if kind == "path" else 64), Hkv=Hkv,
                 N=_log_int(rng, 1, 1024 if kind == "path" else 32768),
                 bits=rng.choice(("int4", "mixed")), ragged=rng.random() < 0.5)
        if kind == "select":  # from more groups than are taken
            c["N"] = _log_int(rng, 1024, 32768)
            c.update(Hq=Hq, k=_log_int(rng, 8, min(128, c["N"] // 128)))
        if kind == "selected":
            c.update(Hq=Hq, k=_log_int(rng, 1, 128))
        if kind == "tree":
            c.update(Hq=Hq, T=_log_int(rng, 1, 256), chain=rng.random() < 0.3)
        if kind == "path":
            c.update(T=_log_int(rng, 1, 256), P=_log_int(rng, 1, 32))
        w = work(c)
        if w["bytes"] <= MAX_BYTES and w["flops"] <= MAX_FLOPS and c["B"] * Hkv * c["N"] <= MAX_CACHE:
            return c


# ---- inputs ------------------------------------------------------------------
def _gen(*key):
    s = 0x5EED
    for k in key:
        s = (s * 1000003 + int(k) + 1) % (2 ** 62)
    return torch.Generator(device="cuda").manual_seed(s)


def _randn(shape, *key):
    return torch.randn(*shape, generator=_gen(*key), device="cuda", dtype=torch.float16)


def _head_bits(c):
    bits = [4] * c["Hkv"]
    if c["bits"] == "mixed":
        for h in random.Random(c["Hkv"]).sample(range(c["Hkv"]), c["Hkv"] // 2):
            bits[h] = 2
    return bits


def _lengths(c):
    """Cached tokens of each sequence: N, or spread up to N."""
    if not c["ragged"]:
        return [c["N"]] * c["B"]
    rng = random.Random(c["B"] * 1000003 + c["N"])
    n = [c["N"]] + [_log_int(rng, max(1, c["N"] // 64), c["N"]) for _ in range(c["B"] - 1)]
    rng.shuffle(n)
    return n


def _max_groups(c):
    return max(_lengths(c)) // GROUP + 1


def _tree_lens(c):
    """Nodes of each sequence's tree: T, or spread up to T where lengths are."""
    if not c.get("ragged", c["B"] > 1):
        return [c["T"]] * c["B"]
    rng = random.Random(c["B"] * 7919 + c["T"])
    n = [c["T"]] + [rng.randint(max(1, c["T"] // 4), c["T"]) for _ in range(c["B"] - 1)]
    rng.shuffle(n)
    return n


def _gain(u, Hkv, *key):
    """Channel gains of the keys of u sequences [u][Hkv][128]: four channels at 10."""
    gain = torch.ones(u, Hkv, D, device="cuda")
    ch = torch.rand(u, Hkv, D, generator=_gen(*key), device="cuda").argsort(dim=-1)[..., :4]
    return gain.scatter_(-1, ch, 10.0)


def _step2(x8, levels):
    """(codes, s, z) of int8 values [.., Hkv, 64, 128], per channel."""
    z = x8.amin(-2)
    s = torch.clamp(torch.ceil((x8.amax(-2) - z) / levels), min=1.0)
    su = s.unsqueeze(-2)
    return torch.floor((2 * (x8 - z.unsqueeze(-2)) + su) / (2 * su)), s, z


def _pack(codes, bits):
    """Codes [.., n] to bytes [.., n * bits / 8], the first in the low bits."""
    x = codes.to(torch.uint8).unflatten(-1, (-1, 8 // bits))
    w = torch.tensor([1 << (bits * i) for i in range(8 // bits)], dtype=torch.uint8, device="cuda")
    return (x * w).sum(-1, dtype=torch.uint8)


def _offsets(bits):
    off = [0]
    for b in bits:
        off.append(off[-1] + 512 * b)
    return off


def _fill(c, seed):
    """A cache filled as by a prefill of each sequence, and the buffer behind it."""
    B, Hkv, bits, lens = c["B"], c["Hkv"], _head_bits(c), _lengths(c)
    mg, off = _max_groups(c), _offsets(bits)
    g = _gen(seed, 2)
    bt = torch.randperm(B * 4 * mg, generator=g, device="cuda").to(torch.int32).view(B, 4 * mg)
    gt = torch.randperm(B * mg, generator=g, device="cuda").to(torch.int32).view(B, mg)
    pages = torch.zeros(B * 4 * mg, off[-1], dtype=torch.uint8, device="cuda")
    meta = torch.zeros(B * mg, Hkv, 4, D, dtype=torch.int8, device="cuda")
    scale = torch.zeros(B * mg, Hkv, 2, device="cuda")
    gain = _gain(B, Hkv, seed, 3)
    levels = torch.tensor([(1 << b) - 1.0 for b in bits], device="cuda").view(1, Hkv, 1)
    seq = torch.tensor(lens, device="cuda")
    ng = seq // GROUP
    b_of = torch.repeat_interleave(torch.arange(B, device="cuda"), ng)
    g_of = torch.arange(len(b_of), device="cuda") - (ng.cumsum(0) - ng)[b_of]
    top = torch.zeros(B, Hkv, 2, device="cuda")
    step = max(1, (1 << 25) // (Hkv * GROUP * D))
    for at in range(0, len(b_of), step):
        b, gr = b_of[at:at + step], g_of[at:at + step]
        slot, pg = gt[b, gr].long(), bt.view(B, mg, 4)[b, gr].long()
        for which in (0, 1):
            x = torch.randn(len(b), Hkv, GROUP, D, generator=_gen(seed, 4, at, which), device="cuda")
            if which == 0:
                x *= gain[b].unsqueeze(-2)
            s1 = x.abs().amax((-2, -1)) / QMAX
            codes, s, z = _step2(torch.round(x / s1[..., None, None]), levels)
            scale[slot, :, which] = s1
            meta[slot, :, 2 * which] = s.to(torch.uint8).view(torch.int8)
            meta[slot, :, 2 * which + 1] = z.to(torch.int8)
            top[:, :, which].scatter_reduce_(0, b[:, None].expand(-1, Hkv), s1, "amax")
            codes = codes.view(len(b), Hkv, 4, PAGE, D)
            if which == 1:
                codes = codes.transpose(-1, -2)
            for h in range(Hkv):
                o = off[h] + 256 * bits[h] * which
                pages[pg, o:o + 256 * bits[h]] = _pack(codes[:, h].flatten(-2), bits[h])
    rows = torch.arange(GROUP, device="cuda")
    k = torch.randn(B, Hkv, GROUP, D, generator=_gen(seed, 5), device="cuda") * gain.unsqueeze(-2)
    v = torch.randn(B, Hkv, GROUP, D, generator=_gen(seed, 6), device="cuda")
    live = (rows < (seq % GROUP)[:, None])[:, None, :, None]
    part = torch.stack([(x * live).abs().amax((-2, -1)) / QMAX for x in (k, v)], -1)
    top = torch.where(ng[:, None, None] > 0, top, torch.where(part > 0, part, part.amax() + 0.02))
    k8, v8 = (torch.where(live, torch.round(x / top[:, :, i, None, None]).clamp(-QMAX, QMAX), 0.0)
              for i, x in enumerate((k, v)))
    return dict(B=B, Hkv=Hkv, mg=mg, bits=bits, pages=pages, meta=meta, scale=scale, bt=bt, gt=gt,
                gain=gain, seq=seq.to(torch.int32), levels=levels, tk=k8.to(torch.int8),
                tv=v8.transpose(-1, -2).contiguous().to(torch.int8), tscale=top, **_layout(bits))


def _layout(bits):
    """Byte in a page and shift of every code: K [Hkv][16][128], V [Hkv][16][128]."""
    b = torch.tensor(bits, device="cuda").view(-1, 1, 1)
    off = torch.tensor(_offsets(bits)[:-1], device="cuda").view(-1, 1, 1)
    t = torch.arange(PAGE, device="cuda").view(1, -1, 1)
    ch = torch.arange(D, device="cuda").view(1, 1, -1)
    kbit, vbit = (t * D + ch) * b, (ch * PAGE + t) * b
    return dict(kbyte=off + kbit // 8, kshift=(kbit % 8).to(torch.uint8),
                vbyte=off + 256 * b + vbit // 8, vshift=(vbit % 8).to(torch.uint8),
                cmask=((1 << b) - 1).to(torch.uint8))


def _parents(c, seed):
    """Parents [B][T] of random trees, or of chains."""
    B, T = c["B"], c["T"]
    i = torch.arange(T, device="cuda")
    u = torch.rand(B, T, generator=_gen(seed, 8), device="cuda")
    p = torch.minimum((u * (i + 1)).floor().long(), i) - 1
    return (i - 1).expand(B, T).to(torch.int32).contiguous() if c.get("chain") else p.to(torch.int32)


def _ancestors(parents, lens):
    """Ancestor matrix [B][T][T] and depths [B][T] on the host, node by node."""
    p = parents.cpu().numpy()
    B, T = p.shape
    see = np.zeros((B, T, T), bool)
    depth = np.full((B, T), -1, np.int32)
    for i in range(T):
        live = np.asarray(lens) > i
        up = np.where(live & (p[:, i] >= 0))[0]
        see[up, i] = see[up, p[up, i]]
        see[live, i, i] = True
        depth[live, i] = 0
        depth[up, i] = depth[up, p[up, i]] + 1
    return see, depth


def _mask_words(see):
    """Bits [B][T][ceil(T / 64)] as int64 of a truth matrix [B][T][T]."""
    B, T, _ = see.shape
    W = (T + 63) // 64
    bits = np.zeros((B, T, 64 * W), bool)
    bits[:, :, :T] = see
    words = np.packbits(bits, axis=-1, bitorder="little").view(np.int64).reshape(B, T, W)
    return torch.from_numpy(words).cuda()


def _handles(s):
    """The cache and buffer objects that a program keeps beside its tensors."""
    import paper_2412_08585_amd as ta
    cache = ta.PagedKVCache(1, 1, s["bits"])
    cache.pages, cache.group_meta, cache.group_scale = s["pages"], s["meta"], s["scale"]
    tail = ta.KVTail(1, s["Hkv"])
    tail.batch, tail.k, tail.v, tail.scale = s["B"], s["tk"], s["tv"], s["tscale"]
    return dict(ta=ta, cache=cache, tail=tail)


def prepare(c, seed):
    kind, B = c["kind"], c["B"]
    if kind == "mask":
        s = dict(c=c, parents=_parents(c, seed),
                 lens=torch.tensor(_tree_lens(c), dtype=torch.int32, device="cuda"))
        if own:
            import paper_2412_08585_amd as ta
            s["ta"] = ta
        return s
    s = dict(c=c, **_fill(c, seed))
    if own:
        s.update(_handles(s))
    Hkv = c["Hkv"]
    if kind in ("select", "selected"):
        s["q"] = _randn((B, c["Hq"], D), seed, 7)
        s["G"] = c["Hq"] // Hkv
        if kind == "select":
            if own:
                s["ws"] = s["ta"].select_workspace(B, c["Hq"], s["mg"])
            return s
        # a choice as a score would make it: distinct groups in ascending order
        ng = (s["seq"] // GROUP).view(B, 1, 1)
        g = torch.arange(s["mg"], device="cuda")
        u = torch.rand(B, Hkv, s["mg"], generator=_gen(seed, 9), device="cuda")
        u = torch.where(g < ng, u, 2.0)
        keep = torch.sort(u, -1)[1][..., :c["k"]]
        keep = torch.sort(torch.where(keep < ng, keep, s["mg"]), -1)[0]
        sel = torch.full((B, Hkv, c["k"]), -1, dtype=torch.int32, device="cuda")
        sel[..., :keep.shape[-1]] = torch.where(keep < ng, keep, -1)
        s["sel"] = sel
        if own:
            s["ws"] = s["ta"].selected_workspace(B, c["Hq"], Hkv, c["k"], with_tail=True)
        return s
    T = c["T"]
    lens = _tree_lens(c)
    s["tlen"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["k_tree"] = (torch.randn(B, Hkv, T, D, generator=_gen(seed, 10), device="cuda")
                   * s["gain"].unsqueeze(-2)).half()
    s["v_tree"] = _randn((B, Hkv, T, D), seed, 11)
    parents = _parents(c, seed)
    see, depth = _ancestors(parents, lens)
    if kind == "tree":
        s["G"] = c["Hq"] // Hkv
        s["q"] = _randn((B, c["Hq"], T, D), seed, 7)
        s["mask"] = _mask_words(see)
        # rows behind a tree's last node stay as they are
        s["o"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(B, c["Hq"], T, device="cuda")
        if own:
            s["ws"] = s["ta"].tree_workspace(B, c["Hq"], Hkv, T, s["mg"], with_tail=True)
        return s
    # a path from a root to a random node, cut where it fills the buffer: the
    # same pass can be made again on what it leaves
    P = c["P"]
    rng = random.Random(seed * 31 + B)
    path, plen = np.full((B, P), -1, np.int32), np.zeros(B, np.int32)
    for b, n in enumerate(_lengths(c)):
        node = max((rng.randrange(lens[b]) for _ in range(4)), key=lambda x: depth[b, x])
        nodes = np.nonzero(see[b, node])[0][:min(P, GROUP - n % GROUP)]
        path[b, :len(nodes)], plen[b] = nodes, len(nodes)
    s["path"], s["plen"] = torch.from_numpy(path).cuda(), torch.from_numpy(plen).cuda()
    return s


# ---- one pass ------------------------------------------------------------------
def run(s):
    kind = s["c"]["kind"]
    if own:
        return _run_own(kind, s)
    if kind == "select":
        return _select(s)
    if kind == "selected":
        return _selected(s)
    if kind == "mask":
        return _mask(s)
    return _tree(s) if kind == "tree" else _path(s)


def _run_own(kind, s):
    ta = s["ta"]
    if kind == "mask":
        mask, depth = ta.turbo_tree_mask(s["parents"], s["lens"])
        return dict(mask=mask, depth=depth)
    if kind == "select":
        return dict(sel=ta.turbo_select_groups(s["q"], s["cache"], s["seq"], s["bt"], s["gt"],
                                               s["c"]["k"], keep_first=FIRST, keep_last=LAST,
                                               workspace=s["ws"]))
    if kind == "selected":
        o, lse = ta.turbo_attn_selected(s["q"], s["cache"], s["seq"], s["bt"], s["gt"], s["sel"],
                                        tail=s["tail"], workspace=s["ws"], return_lse=True)
        return dict(o=o, lse=lse)
    if kind == "tree":
        o, lse = ta.turbo_attn_tree(s["q"], s["k_tree"], s["v_tree"], s["mask"], s["tlen"],
                                    s["cache"], s["seq"], s["bt"], s["gt"], tail=s["tail"],
                                    workspace=s["ws"], out=s["o"], lse_out=s["lse"])
        return dict(o=o, lse=lse)
    ta.turbo_append_path(s["k_tree"], s["v_tree"], s["path"], s["plen"], s["seq"], s["cache"],
                         s["tail"], s["bt"], s["gt"])
    return _path_state(s)


def _path_state(s):
    """The buffer's codes and the cache, as they are held: whole numbers, and scales."""
    return dict(k=s["tk"], v=s["tv"], pages=s["pages"], meta=s["meta"], scale=s["scale"])


# ---- plain forms ---------------------------------------------------------------
def _quantized(q):
    """int8 codes (as fp32) and scale of the rows of q: nearest integers of the
    product with 119 / max rounded to binary32, which 64 bits hold exactly."""
    top = q.float().abs().amax(-1, keepdim=True)
    inv = torch.where(top > 0, QMAX / top, 0.0)
    return torch.round(q.double() * inv.double()).clamp(-QMAX, QMAX).float(), top / QMAX


def _select(s):
    B, Hkv, G, mg, k = s["B"], s["Hkv"], s["G"], s["mg"], s["c"]["k"]
    q8, sq = _quantized(s["q"].view(B, Hkv, G, D))
    slot = s["gt"].long()
    m = s["meta"][slot]                                          # [B][mg][Hkv][4][128]
    step = m[..., 0, :].view(torch.uint8).float() * s["levels"]
    # whole numbers below 2^24: exact in fp32 in any order
    sums = torch.matmul(q8, m[..., 1, :].float().permute(0, 2, 3, 1))
    sums = sums + torch.matmul(q8.clamp(min=0), step.permute(0, 2, 3, 1))
    bound = sums * sq * s["scale"][slot][..., 0].transpose(1, 2).unsqueeze(2)
    ng = (s["seq"] // GROUP).clamp(max=mg).view(B, 1, 1)
    g = torch.arange(mg, device=slot.device)
    live = g < ng
    bound = torch.where(live.unsqueeze(2), bound, -math.inf)
    score = (bound - bound.amax(-1, keepdim=True)).amax(2)
    score = torch.where(live & ((g < FIRST) | (g >= ng - LAST)), math.inf, score)
    score = torch.where(live, score, -math.inf)
    best = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :k]
    best = torch.sort(torch.where(best < ng, best, mg), -1)[0]
    sel = torch.full((B, Hkv, k), -1, dtype=torch.int32, device=slot.device)
    sel[..., :best.shape[-1]] = torch.where(best < mg, best, -1)
    return dict(sel=sel)


def _values(s, pg, slot):
    """fp32 keys and values [B][Hkv][64 n][128] of groups: pg [B][Hkv][n][4] pages,
    slot [B][Hkv][n]."""
    flat = s["pages"].view(-1)
    base = pg[..., None, None] * s["pages"].shape[1]
    h = torch.arange(s["Hkv"], device=pg.device).view(1, -1, 1)
    m, sc = s["meta"][slot, h], s["scale"][slot, h]
    mask = s["cmask"][:, None, None]
    k = ((flat[base + s["kbyte"][:, None, None]] >> s["kshift"][:, None, None]) & mask).float()
    k = k.flatten(3, 4) * m[..., 0:1, :].view(torch.uint8).float() + m[..., 1:2, :].float()
    v = ((flat[base + s["vbyte"][:, None, None]] >> s["vshift"][:, None, None]) & mask).float()
    v = v.flatten(3, 4) * m[..., 2:3, :].view(torch.uint8).float() + m[..., 3:4, :].float()
    return (k * sc[..., 0, None, None]).flatten(2, 3), (v * sc[..., 1, None, None]).flatten(2, 3)


def _buffered(s):
    """fp32 keys and values [B][Hkv][64][128] of the buffer, and which rows are live."""
    k = s["tk"].float() * s["tscale"][..., 0, None, None]
    v = s["tv"].transpose(-1, -2).float() * s["tscale"][..., 1, None, None]
    return k, v, torch.arange(GROUP, device=k.device) < (s["seq"] % GROUP).view(-1, 1, 1, 1)


def _attend(q, k, v, live):
    """softmax(q k^T / sqrt(128)) v over the live tokens, and log-sums; rows that
    see none give 0 and -inf."""
    x = torch.where(live, torch.matmul(q.float(), k.transpose(-1, -2)) / math.sqrt(D), -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.where(live, torch.exp(x - m), 0.0)
    l = p.sum(-1, keepdim=True)
    o = torch.where(l > 0, torch.matmul(p, v) / l, 0.0)
    return o, torch.where(l > 0, m + torch.log(l), -math.inf)[..., 0]


def _selected(s):
    B, Hkv, G, mg, sel = s["B"], s["Hkv"], s["G"], s["mg"], s["sel"]
    ng = (s["seq"] // GROUP).clamp(max=mg).view(B, 1, 1)
    ok = (sel >= 0) & (sel < ng)
    g = torch.where(ok, sel, 0).long()
    b = torch.arange(B, device=g.device).view(B, 1, 1)
    k, v = _values(s, s["bt"].view(B, mg, 4)[b, g].long(), s["gt"][b, g].long())
    tk, tv, tl = _buffered(s)
    live = torch.cat([ok.repeat_interleave(GROUP, -1).unsqueeze(2), tl.expand(-1, Hkv, -1, -1)], -1)
    o, lse = _attend(s["q"].view(B, Hkv, G, D), torch.cat([k, tk], 2), torch.cat([v, tv], 2), live)
    return dict(o=o.view(B, Hkv * G, D).half(), lse=lse.view(B, Hkv * G))


def _mask(s):
    p, lens = s["parents"].long(), s["lens"].view(-1, 1)
    B, T = p.shape
    i = torch.arange(T, device=p.device)
    live = i < lens
    see = torch.eye(T, dtype=torch.bool, device=p.device).expand(B, T, T)
    up = torch.where(live, p, -1)
    for _ in range(T.bit_length()):  # ancestors within 1, 2, 4, .. steps
        at = up.clamp(min=0)
        far = torch.gather(see, 1, at.unsqueeze(-1).expand(B, T, T)) & (up >= 0).unsqueeze(-1)
        see = see | far
        up = torch.where(up >= 0, torch.gather(up, 1, at), -1)
    see = see & live.unsqueeze(-1)
    W = (T + 63) // 64
    bit = torch.nn.functional.pad(see.long(), (0, 64 * W - T)).view(B, T, W, 64)
    words = (bit << torch.arange(64, device=p.device)).sum(-1)
    return dict(mask=words, depth=(see.sum(-1) - 1).to(torch.int32))


def _tree(s):
    B, Hkv, G, mg, T = s["B"], s["Hkv"], s["G"], s["mg"], s["c"]["T"]
    pg = s["bt"].view(B, 1, mg, 4).expand(-1, Hkv, -1, -1).long()
    k, v = _values(s, pg, s["gt"].view(B, 1, mg).expand(-1, Hkv, -1).long())
    tk, tv, tl = _buffered(s)
    i = torch.arange(T, device=k.device)
    tlen = s["tlen"].view(B, 1, 1)
    see = (s["mask"][:, :, i // 64] >> (i % 64)) & 1 != 0
    see = see & (i < tlen)
    cached = torch.arange(mg * GROUP, device=k.device) < (s["seq"] // GROUP * GROUP).view(B, 1, 1, 1)
    live = torch.cat([cached.expand(-1, 1, T, -1), tl.expand(-1, 1, T, -1), see.unsqueeze(1)], -1)
    q = s["q"].view(B, Hkv, G * T, D)
    o, lse = _attend(q, torch.cat([k, tk, s["k_tree"].float()], 2),
                     torch.cat([v, tv, s["v_tree"].float()], 2), live.repeat(1, 1, G, 1))
    row = i < tlen
    return dict(o=torch.where(row.view(B, 1, T, 1), o.view(B, Hkv * G, T, D).half(), s["o"]),
                lse=torch.where(row, lse.view(B, Hkv * G, T), s["lse"]))


def _codes(x, scale):
    """Codes of the buffer: products with the scale's inverse in binary32, in 64 bits."""
    inv = torch.where(scale > 0, 1.0 / scale, 0.0).double()
    return torch.round(x.double() * inv).clamp(-QMAX, QMAX)


def _path(s):
    B, Hkv, mg, bits = s["B"], s["Hkv"], s["mg"], s["bits"]
    node = s["path"].clamp(min=0).long()
    i = torch.arange(node.shape[1], device=node.device)
    at = node.view(B, 1, -1, 1).expand(-1, Hkv, -1, D)
    k = _codes(torch.gather(s["k_tree"], 2, at), s["tscale"][..., 0, None, None])
    v = _codes(torch.gather(s["v_tree"], 2, at), s["tscale"][..., 1, None, None])
    start = s["seq"] % GROUP
    b, j = torch.nonzero(i < s["plen"].view(B, 1), as_tuple=True)
    row = start[b].long() + j
    s["tk"][b, :, row] = k[b, :, j].to(torch.int8)
    s["tv"][b, :, :, row] = v[b, :, j].to(torch.int8)
    full = torch.nonzero(start + s["plen"] == GROUP)[:, 0]
    g = (s["seq"] // GROUP)[full].long()
    slot, pg = s["gt"][full, g].long(), s["bt"].view(B, mg, 4)[full, g].long()
    x8 = torch.stack([s["tk"][full], s["tv"][full].transpose(-1, -2)]).float()
    codes, step, zero = _step2(x8, s["levels"])
    s["meta"][slot] = torch.stack([step[0].to(torch.uint8).view(torch.int8), zero[0].to(torch.int8),
                                   step[1].to(torch.uint8).view(torch.int8), zero[1].to(torch.int8)], 2)
    s["scale"][slot] = s["tscale"][full]
    codes = codes.to(torch.uint8).view(2, len(full), Hkv, 4, PAGE, D)
    flat = torch.zeros(len(full), 4, s["pages"].shape[1], dtype=torch.uint8, device=pg.device)
    for which, byte, shift in ((0, s["kbyte"], s["kshift"]), (1, s["vbyte"], s["vshift"])):
        put = (codes[which].transpose(1, 2) << shift).flatten(2)
        flat.scatter_add_(2, byte.flatten().expand(len(full), 4, -1), put)
    s["pages"][pg.flatten()] = flat.view(-1, flat.shape[-1])
    return _path_state(s)


# ---- what a pass cannot do without -----------------------------------------------
def _group_bytes(c):
    """Bytes of one cached group over all KV heads: codes, s and z, block scales."""
    return sum(2 * GROUP * D * b // 8 + 4 * D + 8 for b in _head_bits(c))


def work(c):
    kind, B = c["kind"], c["B"]
    if kind == "mask":
        return dict(bytes=4.0 * B * c["T"] + B * c["T"] * (8.0 * ((c["T"] + 63) // 64) + 4),
                    flops=float(B) * c["T"] * ((c["T"] + 63) // 64))
    Hkv, lens = c["Hkv"], _lengths(c)
    tables = 20.0
    if kind == "path":
        # a path of a random tree of T nodes is about log T nodes long
        n = min(c["P"], math.ceil(math.log(c["T"])) + 1) * B
        return dict(bytes=n * Hkv * D * 6.0, flops=4.0 * n * Hkv * D)
    Hq = c["Hq"]
    io = 4.0 * B * Hq * D + 4.0 * B * Hq
    if kind == "select":
        groups = sum(n // GROUP for n in lens)
        return dict(bytes=2.0 * B * Hq * D + groups * (Hkv * (2 * D + 4) + tables) + 4.0 * B * Hkv * c["k"],
                    flops=4.0 * D * Hq * groups)
    buffered = sum(2.0 * (n % GROUP) * Hkv * D for n in lens)
    if kind == "selected":
        groups = sum(min(c["k"], n // GROUP) for n in lens)
        tokens = GROUP * groups + sum(n % GROUP for n in lens)
        return dict(bytes=io + groups * (_group_bytes(c) + 4.0 * Hkv) + buffered, flops=4.0 * D * Hq * tokens)
    T = _tree_lens(c)
    groups = sum(n // GROUP for n in lens)
    nbytes = groups * (_group_bytes(c) + tables) + buffered
    nbytes += sum(4.0 * t * (Hq + Hkv) * D + 4.0 * t * Hq + 8.0 * t * ((c["T"] + 63) // 64) for t in T)
    return dict(bytes=nbytes, flops=sum(4.0 * D * Hq * t * (n + t) for n, t in zip(lens, T)))


# ---- the same results in 64 bits ----------------------------------------------
def _unpacked(s, b, h, groups):
    """fp64 keys and values [64 n][128] of groups of (sequence b, KV head h)."""
    bits, off = s["bits"][h], _offsets(s["bits"])[h]
    pg = s["bt"][b].view(-1, 4)[groups].long()                   # [n][4]
    slot = s["gt"][b][groups].long()
    region = s["pages"][:, off:off + 512 * bits][pg]  # [n][4][512 bits]
    codes = torch.stack([(region >> (bits * i)) & ((1 << bits) - 1) for i in range(8 // bits)], -1)
    codes = codes.flatten(-2).double().reshape(-1, 4, 2, PAGE * D)
    k = codes[:, :, 0].reshape(-1, GROUP, D)
    v = codes[:, :, 1].reshape(-1, 4, D, PAGE).transpose(-1, -2).reshape(-1, GROUP, D)
    m, sc = s["meta"][slot, h].long(), s["scale"][slot, h].double()
    k = (k * (m[:, 0:1] & 255) + m[:, 1:2]) * sc[:, 0].view(-1, 1, 1)
    v = (v * (m[:, 2:3] & 255) + m[:, 3:4]) * sc[:, 1].view(-1, 1, 1)
    return k.reshape(-1, D), v.reshape(-1, D)


def _exact_rows(s, b, h, q, groups, more=None, see=None):
    """(o, lse) in fp64 of query rows q over groups, the buffer, and more (k, v)
    of which row i sees see[i]."""
    k, v = _unpacked(s, b, h, groups)
    nt = int(s["seq"][b]) % GROUP
    tk = s["tk"][b, h, :nt].double() * s["tscale"][b, h, 0].double()
    tv = s["tv"][b, h, :, :nt].t().double() * s["tscale"][b, h, 1].double()
    k, v = torch.cat([k, tk]), torch.cat([v, tv])
    live = torch.ones(len(q), len(k), dtype=torch.bool, device=q.device)
    if more is not None:
        k, v, live = torch.cat([k, more[0].double()]), torch.cat([v, more[1].double()]), torch.cat([live, see], 1)
    x = (q.double() @ k.t()) / math.sqrt(D)
    x = x.masked_fill(~live, -math.inf)
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - lse.masked_fill(lse == -math.inf, 0.0)[:, None])
    return p @ v, lse


def _exact_select(s):
    B, Hkv, G, k = s["B"], s["Hkv"], s["G"], s["c"]["k"]
    sel = np.full((B, Hkv, k), -1, np.int32)
    q = s["q"].cpu().numpy().reshape(B, Hkv, G, D)
    for b in range(B):
        ng = int(s["seq"][b]) // GROUP
        slot = s["gt"][b, :ng].long()
        m, sc = s["meta"][slot].cpu().numpy(), s["scale"][slot].cpu().numpy()
        for h in range(Hkv):
            top = np.abs(q[b, h].astype(np.float32)).max(-1)
            inv = (np.float32(QMAX) / top).astype(np.float64)
            codes = np.rint(q[b, h].astype(np.float64) * inv[:, None]).astype(np.int64)
            z, st = m[:, h, 1].astype(np.int64), m[:, h, 0].view(np.uint8).astype(np.int64)
            i = codes @ z.T + ((1 << s["bits"][h]) - 1) * (np.maximum(codes, 0) @ st.T)
            # the definition's roundings: of the sum times s_q, of that times s_K, of the difference
            bound = (i.astype(np.float32) * (top / np.float32(QMAX))[:, None]) * sc[None, :, h, 0]
            if ng == 0:
                continue
            score = (bound - bound.max(1, keepdims=True)).max(0)
            order = sorted(range(ng), key=lambda g: (not (g < FIRST or g >= ng - LAST), -score[g], g))
            best = sorted(order[:k])
            sel[b, h, :len(best)] = best
    return dict(sel=torch.from_numpy(sel).cuda())


def exact(c, seed):
    s = prepare(c, seed)
    kind = c["kind"]
    if kind == "mask":
        see, depth = _ancestors(s["parents"], _tree_lens(c))
        return dict(mask=_mask_words(see), depth=torch.from_numpy(depth).cuda())
    if kind == "select":
        return _exact_select(s)
    if kind == "path":
        full = (s["seq"] % GROUP + s["plen"] == GROUP).nonzero()[:, 0]
        scale = s["scale"].double()
        scale[s["gt"][full, s["seq"][full] // GROUP].long()] = s["tscale"][full].double()
        return dict(k=None, v=None, pages=None, meta=None, scale=scale)
    B, Hq, Hkv, G = c["B"], c["Hq"], c["Hkv"], s["G"]
    if kind == "selected":
        o = torch.zeros(B, Hq, D, dtype=torch.float64, device="cuda")
        lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device="cuda")
        for b in range(B):
            for h in range(Hkv):
                groups = s["sel"][b, h]
                rows = slice(h * G, h * G + G)
                o[b, rows], lse[b, rows] = _exact_rows(s, b, h, s["q"][b, rows], groups[groups >= 0].long())
        return dict(o=o, lse=lse)
    T = c["T"]
    o = torch.zeros(B, Hq, T, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(B, Hq, T, dtype=torch.float64, device="cuda")
    bit = torch.arange(64, device="cuda")
    for b, t in enumerate(_tree_lens(c)):
        see = ((s["mask"][b].unsqueeze(-1) >> bit) & 1).flatten(1).bool()[:t, :t]
        groups = torch.arange(int(s["seq"][b]) // GROUP, device="cuda")
        for h in range(Hkv):
            more = (s["k_tree"][b, h, :t], s["v_tree"][b, h, :t])
            rows = s["q"][b, h * G:h * G + G, :t].reshape(G * t, D)
            ou, lu = _exact_rows(s, b, h, rows, groups, more, see.repeat(G, 1))
            o[b, h * G:h * G + G, :t], lse[b, h * G:h * G + G, :t] = ou.view(G, t, D), lu.view(G, t)
    return dict(o=o, lse=lse)
