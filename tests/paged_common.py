"""Paged caches for the tests, and the operators' definitions in 64 bits on the CPU."""
import math

import torch

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
HALF_STEP = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24, "e4m3": 2.0 ** -4}


class Cache:
    """Pools [n_layers, n_pages, page, hkv, d] (the layer axis left off for one layer) of random rows, NaN in every slot that no
    request's rows fill; pages in random order, -1 in the table behind a request's last page."""

    def __init__(self, seed, lens, hkv, d, kind="bf16", page=16, layout="nhd", n_layers=0, spare_pages=3, room=0, scales=True):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.hkv, self.d, self.kind, self.page = list(lens), hkv, d, kind, page
        counts = [-(-(max(0, n) + room) // page) for n in lens]
        n_pages = sum(counts) + spare_pages
        order = torch.randperm(n_pages, generator=g).to(torch.int32)
        self.table = torch.full((len(lens), max(counts + [0]) + 1), -1, dtype=torch.int32)
        at = 0
        for r, n in enumerate(counts):
            self.table[r, :n] = order[at:at + n]
            at += n
        self.spare = order[at:]
        layers = max(1, n_layers)
        self.k_scale = self.v_scale = None
        if kind == "e4m3" and scales:
            self.k_scale, self.v_scale = (0.005 + 0.02 * torch.rand((layers, hkv), generator=g) for _ in "kv")
        pools = []
        for scale in (self.k_scale, self.v_scale):
            x = torch.randn((layers, n_pages, page, hkv, d), generator=g)
            if scale is not None:
                x = (x / scale[:, None, None, :, None]).clamp(-448, 448)
            x = x.to(TYPES[kind])
            used = torch.zeros((n_pages, page), dtype=torch.bool)
            for r, n in enumerate(lens):
                for s in range(max(0, n)):
                    used[self.table[r, s // page], s % page] = True
            bits = x.view(torch.uint8) if kind == "e4m3" else x
            bits[:, ~used] = 0x7f if kind == "e4m3" else float("nan")
            if layout == "hnd":
                x = x.transpose(2, 3).contiguous().transpose(2, 3)
            pools.append(x)
        self.k, self.v = pools
        if not n_layers:
            self.k, self.v = self.k[0], self.v[0]
            if self.k_scale is not None:
                self.k_scale, self.v_scale = self.k_scale[0], self.v_scale[0]
        self.seq_lens = torch.tensor(lens, dtype=torch.int32)

    def cuda(self):
        """(k_pages, v_pages, block_table, seq_lens) on the GPU, with the pools' layout kept, and the scales as keywords."""
        up = lambda x: x.cuda()
        scales = {} if self.k_scale is None else dict(k_scale=up(self.k_scale), v_scale=up(self.v_scale))
        return (up(self.k), up(self.v), up(self.table), up(self.seq_lens)), scales

    def rows(self, r, which="k", layer=None, n=None):
        """Request r's rows [n, hkv, d] in 64 bits, in the values they stand for."""
        pool, scale = (self.k, self.k_scale) if which == "k" else (self.v, self.v_scale)
        if layer is not None:
            pool, scale = pool[layer], None if scale is None else scale[layer]
        n = max(0, self.lens[r]) if n is None else n
        x = torch.stack([pool[self.table[r, s // self.page], s % self.page].double() for s in range(n)]) if n else torch.zeros((0, self.hkv, self.d)).double()
        return x if scale is None else x * scale.double()[:, None]


def attention(q, k, v, scale=None):
    """One request in 64 bits: q [H, d], k and v [n, hkv, d].  Returns o, lse, and what bounds the errors of o and lse: the
    weights' sum of |v| [H, d], and per head the largest sum of |q k| behind a logit."""
    h, d = q.shape
    hkv = k.shape[1]
    if k.shape[0] == 0:
        return torch.zeros(h, d).double(), torch.full((h,), -math.inf).double(), torch.zeros(h, d).double(), torch.zeros(h).double()
    scale = scale or 1.0 / math.sqrt(d)
    kk, vv = (x.repeat_interleave(h // hkv, dim=1) for x in (k, v))
    s = torch.einsum("hd,nhd->hn", q.double(), kk) * scale
    size = torch.einsum("hd,nhd->hn", q.double().abs(), kk.abs()).amax(dim=1) * scale
    p = torch.softmax(s, dim=1)
    return torch.einsum("hn,nhd->hd", p, vv), torch.logsumexp(s, dim=1), torch.einsum("hn,nhd->hd", p, vv.abs()), size


def attention_tolerance(dtype, kind, o, weight, size, d):
    """A logit is a sum of d products in 32 bits: off by at most (d + 2) 2^-24 of the sum of its terms' sizes (`size`), and the
    scale's roundings, 4 more of them; the weights are off by that much, relatively, in the numerator and again in the sum, and by the
    exponential's 2^-21.  A weight is rounded to bf16 (half a step, 2^-8) for bf16 pools and to fp16 (2^-11, or 2^-40 of the largest
    weight below 2^-29 of it; a head has fewer than 2^14 keys here, so 2^-26 of their sum) for e4m3 ones.  O is rounded once."""
    logits = 2.0 * ((d + 6) * 2.0 ** -24 * size[:, None] + 2.0 ** -21)
    weights = {"bf16": 2.0 ** -8, "e4m3": 2.0 ** -11 + 2.0 ** -26, "fp32": 0.0}[kind]
    sums = 2.0 ** -16  # 32-bit sums over the keys, warps and parts
    return weight * (logits + weights + sums) + HALF_STEP[dtype] * o.abs() * 1.02 + 1e-30


def lse_tolerance(lse, size, d):
    return (d + 6) * 2.0 ** -24 * size + 2.0 ** -18 + 2.0 ** -22 * lse.abs()


def angles(positions, inv_freq, sections):
    """[T, rot/2] in 64 bits."""
    pos = positions.double().reshape(-1, positions.shape[-1])
    axis = torch.arange(len(sections)).repeat_interleave(torch.tensor(sections))
    return pos[axis].T * inv_freq.double()


def rotate(x, angle, interleaved):
    """x [T, heads, d] in 64 bits, and for each element the sum of the sizes of what it is made of."""
    x = x.double()
    half = angle.shape[1]
    y, size = x.clone(), x.abs()
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, size


def stored_tolerance(kind, value, size, scale=None):
    """Sine and cosine in 32 bits of a fraction of a turn in 32 bits: off by 2^-22 at most; products and their sum by three more
    roundings of 2^-24: 2^-21 of the sizes in all.  Then half a step of what is stored (e4m3: of the quotient, 2^-4, or 2^-10 where
    that is subnormal, and the quotient's own rounding)."""
    if kind != "e4m3":
        return 2.0 ** -21 * size + HALF_STEP[kind] * value.abs() * 1.001
    units = 1.0 if scale is None else scale.double()[..., None]
    return (2.0 ** -21 + 2.0 ** -23) * size / units + 2.0 ** -4 * value.abs() / units * 1.001 + 2.0 ** -10
