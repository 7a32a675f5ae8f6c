"""Plain 64-bit forms of the sparse and speculative decoding calls, and caches to
run them on.  Test infrastructure only.

Error bound of an attention row against 64 bits (attend): the kernels take the
products of Q K^T exactly and sum them in binary32, so a score is off by at most
dx = (128 + 8) 2^-24 * sm * sum_c |q_c K_c| (the 8 for the scale, log2 e and the
exponent's own rounding); a probability is then off by 2 dx + 2^-20 relative to the
row's sum (2 dx: its own score's and the sum's), and by half a step of fp16, 2^-11,
as an operand of the second product; the row's sums of n terms by (n / 16 + 64) 2^-24
of their absolute terms (a lane sums 16 tokens of 64, then tiles); the output by half
a step, 2^-11 relative or 2^-25 at least (fp16's smallest step is 2^-24)."""
import numpy as np
import torch

from tests import cache_layout

D = 128
SM = 1 / np.sqrt(D)
F16 = 2.0 ** -11


def rand(shape, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).half()


class Filled:
    """A cache of B sequences (lens tokens) and their buffers, on the GPU, as the
    library's own quantization leaves them; host copies for the references."""

    def __init__(self, ta, dev, lens, bits, seed=0, max_groups=None, tail=True):
        B, Hkv = len(lens), len(bits)
        self.lens, self.bits, self.Hkv, self.B = list(lens), list(bits), Hkv, B
        mg = max(1, max(n // 64 for n in lens) + 1) if max_groups is None else max_groups
        self.mg = mg
        rng = np.random.default_rng(seed)
        self.bt = rng.permutation(B * 4 * mg).astype(np.int32).reshape(B, 4 * mg)
        self.gt = rng.permutation(B * mg).astype(np.int32).reshape(B, mg)
        self.cache = ta.PagedKVCache(B * 4 * mg, B * mg, bits, dev)
        self.tail = ta.KVTail(B, Hkv, dev) if tail else None
        self.btd, self.gtd = torch.from_numpy(self.bt).to(dev), torch.from_numpy(self.gt).to(dev)
        self.sl = torch.tensor(self.lens, dtype=torch.int32, device=dev)
        for b, n in enumerate(lens):
            if n <= 0:
                continue
            n = min(n, 64 * mg + n % 64) if max_groups is not None else n
            k, v = rand((1, Hkv, n, D), 100 * seed + 2 * b), rand((1, Hkv, n, D), 100 * seed + 2 * b + 1)
            k[..., 7] *= 10
            k, v = k.to(dev), v.to(dev)
            _, _, sk, sv = ta.turbo_quantize_kv(k, v, self.cache, self.btd[b:b + 1], self.gtd[b:b + 1])
            if tail:
                ta.turbo_tail_init(k, v, sk, sv, self.tail.narrow(b, 1))
        torch.cuda.synchronize()

    def host(self):
        """Host copies of the cache and the buffer as they are now."""
        c = self.cache
        self.pages, self.meta = c.pages.cpu().numpy(), c.group_meta.cpu().numpy()
        self.scale = c.group_scale.cpu().numpy()
        if self.tail is not None:
            self.tk, self.tv = self.tail.k.cpu().numpy(), self.tail.v.cpu().numpy()
            self.ts = self.tail.scale.cpu().numpy()
        return self

    def groups(self, b):
        return min(max(self.lens[b] // 64, 0), self.mg)

    def valid(self, b, g):
        pg, s = self.bt[b, 4 * g:4 * g + 4], self.gt[b, g]
        return bool((pg >= 0).all() and (pg < self.pages.shape[0]).all() and 0 <= s < self.meta.shape[0])

    def kv(self, b, h, groups):
        """fp64 keys and values of groups (those with valid entries) and the buffer."""
        ks, vs = [np.zeros((0, D))], [np.zeros((0, D))]
        for g in groups:
            if not self.valid(b, g):
                continue
            u = cache_layout.read_unit(self.pages, self.meta, self.scale, self.bits,
                                       self.bt[b:b + 1, 4 * g:4 * g + 4], self.gt[b:b + 1, g:g + 1], 0, h, 1)
            ks.append((u["kc"] * u["ks"].astype(float) + u["kz"]) * float(u["sk"][0]))
            vs.append((u["vc"] * u["vs"].astype(float) + u["vz"]) * float(u["sv"][0]))
        if self.tail is not None:
            nt = min(max(self.lens[b] - 64 * self.groups(b), 0), 63)
            ks.append(self.tk[b, h, :nt].astype(float) * float(self.ts[b, h, 0]))
            vs.append(self.tv[b, h, :, :nt].T.astype(float) * float(self.ts[b, h, 1]))
        return np.concatenate(ks), np.concatenate(vs)


def attend(q, k, v, see=None, sm=SM):
    """(o, lse, bound of o, bound of lse) in 64 bits of rows q [R][128]; row i sees
    the tokens of see[i] (all without see)."""
    R, n = len(q), len(k)
    see = np.ones((R, n), bool) if see is None else see
    o, lse = np.zeros((R, D)), np.full(R, -np.inf)
    to, tl = np.zeros((R, D)), np.zeros(R)
    for i in range(R):
        if not see[i].any():
            continue
        kk, vv = k[see[i]], v[see[i]]
        x = sm * (kk @ q[i])
        dx = 136 * 2.0 ** -24 * sm * (np.abs(kk) @ np.abs(q[i])).max()
        m = x.max()
        p = np.exp(x - m)
        l = p.sum()
        o[i], lse[i] = p @ vv / l, m + np.log(l)
        a = p @ np.abs(vv) / l
        sums = (len(x) / 16 + 64) * 2.0 ** -24
        to[i] = F16 * np.abs(o[i]) + 2.0 ** -25 + a * (F16 + 2 * dx + 2.0 ** -20 + sums)
        # m is held in units of ln 2 with 24 bits; log2 l to some units in the last place
        tl[i] = 2 * dx + 2.0 ** -20 + sums + 2.0 ** -22 * (abs(m) + abs(np.log(l)) + 16)
    return o, lse, to, tl


def words_to_matrix(mask, T):
    """bool [B][T][T] of int64 words [B][T][ceil(T/64)]."""
    m = np.ascontiguousarray(mask).view(np.uint64)
    bits = (m[..., None] >> np.arange(64, dtype=np.uint64)) & np.uint64(1)
    return bits.reshape(*m.shape[:-1], -1)[..., :T].astype(bool)


def matrix_to_words(see):
    B, T, _ = see.shape
    W = (T + 63) // 64
    bits = np.zeros((B, T, 64 * W), bool)
    bits[..., :T] = see
    return np.packbits(bits, axis=-1, bitorder="little").view(np.int64).reshape(B, T, W)


def ancestors(parents, lens):
    """(see bool [B][T][T], depth int32 [B][T]) by walking up from every node."""
    B, T = parents.shape
    see, depth = np.zeros((B, T, T), bool), np.full((B, T), -1, np.int32)
    for b in range(B):
        for i in range(min(max(lens[b], 0), T)):
            j, d = i, 0
            see[b, i, i] = True
            while 0 <= parents[b, j] < j:
                j = parents[b, j]
                see[b, i, j] = True
                d += 1
            depth[b, i] = d
    return see, depth


def select(f, q, num, first, last):
    """turbo_select_groups by its definition: integers, and the binary32 roundings
    it names.  q fp16 [B][Hq][128] (numpy)."""
    B, Hq, _ = q.shape
    G = Hq // f.Hkv
    out = np.full((B, f.Hkv, num), -1, np.int32)
    old = np.seterr(all="ignore")
    for b in range(B):
        ng = f.groups(b)
        live = [g for g in range(ng) if f.valid(b, g)]
        if not live:
            continue
        slot = f.gt[b, live]
        for h in range(f.Hkv):
            z = f.meta[slot, h, 1].astype(np.int64)
            s = f.meta[slot, h, 0].view(np.uint8).astype(np.int64)
            L = (1 << f.bits[h]) - 1
            score = np.full(len(live), -np.inf, np.float32)
            for r in range(G):
                x = q[b, h * G + r].astype(np.float32)
                top = np.abs(x).max()
                inv = np.float32(119) / top if top > 0 else np.float32(0)
                c = np.rint(x.astype(np.float64) * np.float64(inv)).clip(-119, 119).astype(np.int64)
                i = np.maximum(c * z, c * (z + L * s)).sum(-1)
                bound = (i.astype(np.float32) * (top / np.float32(119))) * f.scale[slot, h, 0]
                bound = np.where(np.isnan(bound), np.float32(-np.inf), bound)
                d = bound - bound.max()
                score = np.maximum(score, np.where(np.isnan(d), np.float32(-np.inf), d))
            kept = [not (g < first or g >= ng - last) for g in live]
            order = sorted(range(len(live)), key=lambda j: (kept[j], -score[j], j))
            best = sorted(live[j] for j in order[:num])
            out[b, h, :len(best)] = best
    np.seterr(**old)
    return out
