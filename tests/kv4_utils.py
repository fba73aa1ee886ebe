"""The 4-bit key/value cache's definition in 64 bits, on the CPU and apart from the library: quantiser, pool bytes, attention."""
import numpy as np
import torch

GROUP = 32
MAX_SPAN = 15 * 8160.0


def regions(kv_heads, head_dim, pool_rows):
    pad = lambda n: (n + 255) // 256 * 256  # noqa: E731
    codes, params = pad(kv_heads * pool_rows * head_dim // 2), pad(kv_heads * pool_rows * head_dim // GROUP * 4)
    return codes, params


def quantise(x):
    """x [..., head_dim] (any float type) -> codes int64 [..., head_dim], s and mid float64 [..., groups]."""
    y = x.double().reshape(*x.shape[:-1], -1, GROUP)
    bad = ~torch.isfinite(y).all(-1)
    y = torch.where(bad[..., None], 0.0, y)
    lo, hi = y.min(-1).values, y.max(-1).values
    span = hi - lo
    exponent = torch.frexp(span / 15)[1].double()                    # span / 15 in [2^(e-1), 2^e)
    unit = torch.exp2(torch.clamp(exponent - 8, min=-24))
    s = torch.ceil(span / 15 / unit) * unit
    mid = (lo + 8 * s).float().half().double()
    bad |= (s > MAX_SPAN / 15) | ~torch.isfinite(mid)
    c = torch.round((y - mid[..., None]) / torch.where(s == 0, 1.0, s)[..., None]).clamp(-8, 7) + 8
    c = torch.where(bad[..., None], 0.0, c).long().reshape(x.shape)
    nan = float("nan")
    return c, torch.where(bad, nan, s), torch.where(bad, nan, mid)


def values(codes, s, mid):
    c = codes.double().reshape(*codes.shape[:-1], codes.shape[-1] // GROUP, GROUP) - 8
    return (mid[..., None] + s[..., None] * c).reshape(codes.shape)


class Pool:
    """A pool's bytes on the CPU, as the library lays them out."""

    def __init__(self, raw, kv_heads, head_dim, pool_rows):
        codes, params = regions(kv_heads, head_dim, pool_rows)
        assert raw.numel() == 2 * (codes + params)
        n = kv_heads * pool_rows
        self.codes = [raw[w * codes:w * codes + n * head_dim // 2].view(kv_heads, pool_rows, head_dim // 2) for w in range(2)]
        at = 2 * codes
        self.params = [raw[at + w * params:at + w * params + n * head_dim // 8].view(torch.float16)
                       .view(kv_heads, pool_rows, head_dim // GROUP, 2) for w in range(2)]

    def put(self, which, row, x):
        """x [kv_heads, head_dim]"""
        c, s, mid = quantise(x)
        self.codes[which][:, row] = (c[:, 0::2] | c[:, 1::2] << 4).to(torch.uint8)
        self.params[which][:, row] = torch.stack([s, mid], -1).half()

    def get(self, which, rows):
        """[kv_heads, len(rows), head_dim] float64"""
        b = self.codes[which][:, rows].long()
        c = torch.stack([b & 15, b >> 4], -1).flatten(-2)
        p = self.params[which][:, rows].double()
        return values(c, p[..., 0], p[..., 1])


def attention(q, k, v, limits, scale):
    """q [rows, heads, hd], k and v [kv_heads, keys, hd], row i sees keys < limits[i]; all float64.  Returns out, and a bound of
    what rounding may do to each element without the output's own:
      scores are sums of hd + 5 products in 32 bits, exp is good to 2^-20, both change a weight by their absolute error;
      weights are rounded to binary16 once for the values' product (2^-11), sums of n weights in 32 bits (n 2^-24)."""
    rows, heads, hd = q.shape
    share = heads // k.shape[0]
    out, tol = torch.zeros(rows, heads, hd, dtype=torch.float64), torch.zeros(rows, heads, 1, dtype=torch.float64)
    for h in range(heads):
        kh, vh = k[h // share], v[h // share]
        for i in range(rows):
            n = int(limits[i])
            if n <= 0:
                continue
            x = kh[:n] @ q[i, h] * scale
            out[i, h] = torch.softmax(x, 0) @ vh[:n]
            delta = (hd + 16) * 2.0 ** -24 * float((kh[:n].abs() @ q[i, h].abs()).max()) * scale + 2.0 ** -20
            tol[i, h] = float(vh[:n].abs().max()) * (2 * 2.0 ** -11 + 2 * delta + (n + 64) * 2.0 ** -24)
    return out, tol


def check_attention(got, want, tol, what=""):
    half = torch.finfo(got.dtype).eps / 2
    got = got.double().cpu()
    assert torch.isfinite(got).all(), what
    off = (got - want).abs() - (half * want.abs() + tol + 2.0 ** -25)
    assert off.max() <= 0, "%s: %.3g over the bound" % (what, off.max())
    # element by element the bound is loose for long sequences; roundings are independent, so the whole is closer
    norm = want.norm()
    if norm > 0:
        rel = float((got - want).norm() / norm)
        assert rel <= half + 2 * 2.0 ** -11, "%s: relative error %.3g" % (what, rel)


def paged(lens, page, seed=0, spare=2, extra=1):
    """Page table (pages in random order), number of pages, and the pool rows of every sequence's positions."""
    counts = [-(-n // page) for n in lens]
    order = np.random.RandomState(seed).permutation(sum(counts) + spare)
    table = np.full((len(lens), max(counts + [0]) + extra), -1, dtype=np.int32)
    rows, at = [], 0
    for b, (n, c) in enumerate(zip(lens, counts)):
        table[b, :c] = order[at:at + c] * page
        at += c
        rows.append(np.array([table[b, u // page] + u % page for u in range(n)], dtype=np.int64))
    return table, len(order), rows


def random_pool(kv_heads, head_dim, pool_rows, rows, seed):
    """Pool bytes with quantised random rows where `rows` (lists of pool rows) say, NaN parameters everywhere else."""
    codes, params = regions(kv_heads, head_dim, pool_rows)
    raw = torch.full((2 * (codes + params),), 0xFF, dtype=torch.uint8)
    pool = Pool(raw, kv_heads, head_dim, pool_rows)
    g = torch.Generator().manual_seed(seed)
    every = torch.tensor(np.concatenate([np.asarray(r, dtype=np.int64) for r in rows] + [np.zeros(0, np.int64)]))
    if len(every):
        for which in range(2):
            x = torch.randn(kv_heads, len(every), head_dim, generator=g)
            if which == 0:
                x = x + torch.randn(kv_heads, 1, head_dim, generator=g)
            c, s, mid = quantise(x.half())
            pool.codes[which][:, every] = (c[..., 0::2] | c[..., 1::2] << 4).to(torch.uint8)
            pool.params[which][:, every] = torch.stack([s, mid], -1).half()
    return raw, pool
