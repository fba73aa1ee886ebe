"""The 4-bit key/value cache on the GPU against its definition in 64 bits: what is written (byte for byte), read back, and
attended, at the sizes, masks, strides and page sizes where each can go wrong."""
import numpy as np
import pytest
import torch

import kv4_utils as ku

pytestmark = pytest.mark.gpu

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ll():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2604_23467_amd import binding
    binding.load()
    return binding


def dev(a):
    return torch.as_tensor(a).to("cuda:0")


def ints(a):
    return dev(torch.tensor(np.asarray(a), dtype=torch.int32))


def spread(t, kind):
    """The same rows laid out another way: side by side with others, head-major, or on an odd address."""
    rows, heads, hd = t.shape
    if kind == "fused":
        wide = torch.zeros(rows, heads + 3, hd, dtype=t.dtype, device=t.device)
        wide[:, 2:2 + heads] = t
        return wide[:, 2:2 + heads]
    if kind == "head-major":
        return t.transpose(0, 1).contiguous().transpose(0, 1)
    if kind == "odd":
        flat = torch.zeros(rows * heads * (hd + 3) + 1, dtype=t.dtype, device=t.device)
        view = flat[1:].view(rows, heads, hd + 3)[:, :, :hd]
        view.copy_(t)
        return view
    return t


LAYOUTS = ["plain", "fused", "head-major", "odd"]


# ---- writing ----

def hard_rows(head_dim, dtype, seed):
    """Rows whose groups are hard to quantise: constant, tiny, huge, between two codes, not finite."""
    g = torch.Generator().manual_seed(seed)
    groups = [torch.randn(32, generator=g) * s for s in (1e-7, 1e-5, 1e-3, 0.1, 1.0, 30.0, 5000.0)]
    groups += [torch.full((32,), c) for c in (0.0, 0.1, -3.25, 65504.0, 6e-8)]
    groups += [torch.arange(32.0) % 16, (torch.arange(32.0) % 16) / 2 + 100, torch.arange(32.0) * 0.5,        # borders of codes
               (torch.arange(32.0) % 31) * 2.0 ** -24, 1.0 + (torch.arange(32.0) % 2) * 2.0 ** -7]
    groups += [torch.linspace(-61000, 61000, 32), torch.linspace(-65504, 65504, 32), torch.linspace(0, 65504, 32)]
    for bad in (float("nan"), float("inf"), -float("inf")):
        x = torch.randn(32, generator=g)
        x[int(torch.randint(0, 32, (1,), generator=g))] = bad
        groups.append(x)
    groups += [torch.randn(32, generator=g) * 2.0 ** float(torch.rand(1, generator=g) * 24 - 14) +
               float(torch.randn(1, generator=g)) * 2.0 ** float(torch.rand(1, generator=g) * 16 - 8) for _ in range(400)]
    x = torch.cat(groups).to(dtype)
    n = len(x) // head_dim
    return x[:n * head_dim].view(n, 1, head_dim)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("head_dim", [64, 128])
def test_hard_groups_are_held_as_defined(ll, head_dim, dtype):
    k = hard_rows(head_dim, DTYPES[dtype], 1)
    v = k.flip(0)
    n = k.shape[0]
    raw = torch.zeros(ll.ll_kv4_pool_bytes(1, head_dim, 16, 64), dtype=torch.uint8)
    assert n <= 1024
    want = ku.Pool(raw.clone(), 1, head_dim, 1024)
    for j in range(n):
        want.put(0, j, k[j])
        want.put(1, j, v[j])
    pool = dev(raw)
    cache = ll.KV4Cache(pool, 1, head_dim, 16, 64)
    rows = ll.KV4Rows(ints([n]), ints([[16 * i for i in range(64)]]), max_rows=n)
    ll.ll_kv4_write(cache, rows, dev(k), dev(v))
    got = ku.Pool(pool.cpu(), 1, head_dim, 1024)
    for which in range(2):
        a, b = got.params[which], want.params[which]
        same = (a == b) | (a.isnan() & b.isnan())
        assert same.all(), torch.nonzero(~same)[:5].tolist()
        assert torch.equal(got.codes[which], want.codes[which]), torch.nonzero(got.codes[which] != want.codes[which])[:5].tolist()
    # what is held is as near as the format promises
    x = ku.values(*ku.quantise(k))
    s, mid = (t.repeat_interleave(32, -1) for t in ku.quantise(k)[1:])
    ok = x.isfinite()
    assert ((x - k.double()).abs()[ok] <= (s / 2 + mid.abs() * 2.0 ** -11 + 2.0 ** -25)[ok]).all()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype,head_dim,kv_heads,page", [("f16", 128, 3, 7), ("bf16", 64, 5, 16), ("f16", 64, 1, 1), ("bf16", 128, 4, 64)])
def test_ragged_rows_are_written_where_the_table_says_and_nowhere_else(ll, layout, dtype, head_dim, kv_heads, page):
    m = [3, 0, 1, 40, 5, 2]
    lens = [10, 4, 1, 55, 3, 0]             # the last two have rows in front of position 0
    table, pages, rows = ku.paged(lens, page)
    if page == 7:
        table[3, 1] = -1                    # a page that is not there
        table[3, 2] = pages * page - page + 1
    start = np.concatenate([[0], np.cumsum(m)])
    n = int(start[-1]) + 4                  # rows behind the last sequence
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(n, kv_heads, head_dim, generator=g).to(DTYPES[dtype]) for _ in range(2))
    raw, want = ku.random_pool(kv_heads, head_dim, pages * page, [], 5)
    pool = dev(raw.clone())
    cache = ll.KV4Cache(pool, kv_heads, head_dim, page, pages)
    ll.ll_kv4_write(cache, ll.KV4Rows(ints(lens), ints(table), max_rows=max(m), row_start=ints(start)),
                    spread(dev(k), layout), spread(dev(v), layout))
    for b in range(len(m)):
        for j in range(m[b]):
            u = lens[b] - m[b] + j
            at = table[b, u // page] if u >= 0 else -1
            if u >= 0 and 0 <= at <= pages * page - page:
                want.put(0, at + u % page, k[start[b] + j])
                want.put(1, at + u % page, v[start[b] + j])
    assert torch.equal(pool.cpu(), raw)     # `want` writes into raw


def test_only_max_rows_of_a_sequence_are_looked_at(ll):
    raw, want = ku.random_pool(2, 64, 64, [], 5)
    pool = dev(raw.clone())
    k = torch.randn(9, 2, 64).half()
    cache = ll.KV4Cache(pool, 2, 64, 16, 4)
    ll.ll_kv4_write(cache, ll.KV4Rows(ints([20]), ints([[16, 48]]), max_rows=4, row_start=ints([0, 9])), dev(k), dev(k))
    for j in range(4):
        u = 20 - 9 + j
        for which in range(2):
            want.put(which, [16, 48][u // 16] + u % 16, k[j])
    assert torch.equal(pool.cpu(), raw)


# ---- reading ----

@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype,head_dim,kv_heads,page", [("f16", 128, 3, 7), ("bf16", 64, 5, 16), ("f16", 64, 1, 1), ("bf16", 128, 4, 64)])
def test_rows_read_back(ll, layout, dtype, head_dim, kv_heads, page):
    m, lens = [3, 0, 1, 40, 5], [10, 4, 1, 55, 3]
    table, pages, rows = ku.paged(lens, page)
    raw, pool = ku.random_pool(kv_heads, head_dim, pages * page, rows, 5)
    if page == 16:
        table[3, 2] = -16
    start = np.concatenate([[0], np.cumsum(m)])
    n = int(start[-1]) + 4
    before = torch.full((n, kv_heads, head_dim), 7.0, dtype=DTYPES[dtype])
    outs = [spread(dev(before), layout) for _ in range(2)]
    cache = ll.KV4Cache(dev(raw), kv_heads, head_dim, page, pages)
    ll.ll_kv4_read(cache, ll.KV4Rows(ints(lens), ints(table), max_rows=max(m), row_start=ints(start)), *outs)
    for which in range(2):
        want = before.clone().double()
        for b in range(len(m)):
            for j in range(m[b]):
                u = lens[b] - m[b] + j
                at = table[b, u // page] if u >= 0 else -1
                want[start[b] + j] = pool.get(which, [at + u % page])[:, 0] if at >= 0 else 0.0
        # one rounding to 32 bits, one to the output's type
        half = torch.finfo(DTYPES[dtype]).eps / 2 + 2.0 ** -24
        got = outs[which].cpu().double()
        assert ((got - want).abs() <= half * want.abs() + 2.0 ** -25).all()
        assert torch.equal(got[n - 4:], before.double()[n - 4:])


# ---- attention ----

def attend(ll, dtype, heads, kv_heads, head_dim, page, m, lens, seed=0, layout="plain", ragged=True, new=False, holes=(), scale=0.0,
           qscale=1.0, max_len=0):
    table, pages, rows = ku.paged(lens, page, seed)
    raw, pool = ku.random_pool(kv_heads, head_dim, pages * page, rows, seed)
    for b, i in holes:
        table[b, i] = -1
    start = np.concatenate([[0], np.cumsum(m)])
    n = int(start[-1])
    g = torch.Generator().manual_seed(seed + 1)
    q = (qscale * torch.randn(n, heads, head_dim, generator=g)).to(DTYPES[dtype])
    k, v = (torch.randn(n, kv_heads, head_dim, generator=g).to(DTYPES[dtype]) for _ in range(2))
    dpool = dev(raw.clone())
    cache = ll.KV4Cache(dpool, kv_heads, head_dim, page, pages)
    r = ll.KV4Rows(ints(lens), ints(table), max_rows=max(m), row_start=ints(start) if ragged else None, max_len=max_len)
    out = spread(torch.full((n, heads, head_dim), 9.0, dtype=DTYPES[dtype], device="cuda:0"), layout)
    more = dict(k=spread(dev(k), layout), v=spread(dev(v), layout)) if new else {}
    got = ll.ll_kv4_attention(cache, r, spread(dev(q), layout), out=out, scale=scale, **more)
    assert got is out
    want, tol = torch.zeros(n, heads, head_dim, dtype=torch.float64), torch.zeros(n, heads, 1, dtype=torch.float64)
    for b in range(len(m)):
        there = [u for u in range(lens[b]) if table[b, u // page] >= 0]
        at = [int(table[b, u // page]) + u % page for u in there]
        if new:
            for j in range(m[b]):
                u = lens[b] - m[b] + j
                if u in there:
                    pool.put(0, at[there.index(u)], k[start[b] + j])
                    pool.put(1, at[there.index(u)], v[start[b] + j])
        limits = [sum(u <= lens[b] - m[b] + j for u in there) for j in range(m[b])]
        sl = slice(int(start[b]), int(start[b + 1]))
        want[sl], tol[sl] = ku.attention(q[sl].double(), pool.get(0, at), pool.get(1, at), limits, scale or head_dim ** -0.5)
    ku.check_attention(out, want, tol, "attention")
    if new:
        assert torch.equal(dpool.cpu(), raw)
    return out


@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim,page", [
    ("f16", 4, 4, 64, 16), ("f16", 2, 2, 128, 16), ("bf16", 8, 2, 128, 32), ("f16", 6, 2, 64, 7), ("bf16", 3, 3, 64, 1),
    ("f16", 16, 1, 128, 48), ("f16", 20, 1, 64, 16), ("bf16", 7, 1, 128, 100)])
@pytest.mark.parametrize("new", [False, True])
def test_one_row_a_sequence(ll, dtype, heads, kv_heads, head_dim, page, new):
    lens = [1, 2, 15, 16, 17, 0, 31, 32, 33, 47, 63, 64, 65, 127, 128, 129, 255, 257, 640, 1025]
    attend(ll, dtype, heads, kv_heads, head_dim, page, [1] * len(lens), lens, ragged=False, new=new)


@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim,page,length", [
    ("f16", 2, 2, 128, 16, 9000), ("bf16", 8, 1, 64, 64, 20011), ("f16", 4, 4, 64, 9, 4097), ("f16", 5, 1, 128, 16, 3001)])
def test_few_long_sequences(ll, dtype, heads, kv_heads, head_dim, page, length):
    attend(ll, dtype, heads, kv_heads, head_dim, page, [1, 1, 1], [length, 3, length // 2 + 1], ragged=False, new=True)


@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim,page", [
    ("f16", 2, 2, 128, 16), ("f16", 4, 4, 64, 7), ("bf16", 8, 2, 128, 32), ("bf16", 6, 1, 64, 1), ("f16", 3, 1, 128, 24)])
@pytest.mark.parametrize("new", [False, True])
def test_many_rows_a_sequence(ll, dtype, heads, kv_heads, head_dim, page, new):
    m = [1, 2, 5, 16, 17, 33, 0, 64, 100, 130, 3]
    lens = [200, 2, 90, 16, 300, 33, 10, 65, 333, 140, 1]      # the last sequence: two rows in front of position 0
    attend(ll, dtype, heads, kv_heads, head_dim, page, m, lens, new=new)


@pytest.mark.parametrize("rows", [2, 3, 8, 15, 31, 32, 63, 65, 127, 129, 200])
def test_row_counts_around_the_tiles(ll, rows):
    attend(ll, "f16", 2, 1, 128, 16, [rows, rows], [rows, rows + 77], ragged=False)
    attend(ll, "bf16", 1, 1, 64, 16, [rows], [rows + 500], ragged=False)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("head_dim", [64, 128])
def test_layouts_of_rows(ll, layout, head_dim):
    attend(ll, "f16", 4, 2, head_dim, 16, [1, 1, 1], [5, 40, 300], layout=layout, ragged=False, new=True)
    attend(ll, "bf16", 4, 2, head_dim, 16, [30, 1, 70], [30, 40, 300], layout=layout, new=True)


@pytest.mark.parametrize("head_dim", [64, 128])
def test_odd_addresses_in_the_kernels_for_one_and_for_many_rows(ll, head_dim):
    attend(ll, "f16", 3, 3, head_dim, 16, [1, 1, 1], [5, 40, 300], layout="odd", ragged=False, new=True)
    attend(ll, "bf16", 32, 32, head_dim, 16, [65] * 8, [65, 66, 70, 80, 90, 100, 110, 120], layout="odd", ragged=False)


def test_pages_that_are_not_there(ll):
    """Positions without a page are seen by nobody; a row that then sees nothing gives zeros."""
    out = attend(ll, "f16", 2, 2, 128, 16, [1, 1, 1], [100, 20, 40], ragged=False, holes=[(0, 0), (0, 3), (1, 0), (1, 1), (2, 2)])
    assert (out[1] == 0).all()
    out = attend(ll, "f16", 4, 2, 64, 16, [60, 20, 40], [100, 20, 41], holes=[(0, 0), (0, 3), (0, 4), (1, 0), (1, 1), (2, 0)])
    assert (out[60:80] == 0).all() and (out[80:95] == 0).all()


@pytest.mark.parametrize("heads,kv_heads,rows,page", [(2, 2, 1, 16), (2, 2, 1, 7), (8, 1, 2, 16), (8, 2, 3, 7), (32, 32, 65, 16), (32, 32, 65, 7)])
@pytest.mark.parametrize("length", [2 ** 31 - 1, 2 ** 30 + 5, 1100])
def test_lengths_beyond_the_page_table(ll, heads, kv_heads, rows, page, length):
    """All that the table has is seen, by every row, and the rows' own keys have no place."""
    n, seqs = 1024 // page * page, 4 if rows > 64 else 1
    table, pages, at = ku.paged([n] * seqs, page, seed=3, extra=0)
    raw, pool = ku.random_pool(kv_heads, 64, pages * page, at, seed=4)
    g = torch.Generator().manual_seed(5)
    q = torch.randn(seqs * rows, heads, 64, generator=g).half()
    knew = torch.randn(seqs * rows, kv_heads, 64, generator=g).half()
    mem = dev(raw)
    cache = ll.KV4Cache(mem, kv_heads, 64, page, pages)
    layout = ll.KV4Rows(ints([length] * seqs), ints(table), max_rows=rows)
    got = [ll.ll_kv4_attention(cache, layout, dev(q), **new) for new in ({}, dict(k=dev(knew), v=dev(knew)))]
    for b in range(seqs):
        its = slice(b * rows, (b + 1) * rows)
        want, tol = ku.attention(q[its].double(), pool.get(0, at[b]), pool.get(1, at[b]), [n] * rows, 64 ** -0.5)
        for out in got:
            ku.check_attention(out[its], want, tol, "sequence %d" % b)
    assert torch.equal(mem.cpu(), raw)


def test_scales_and_large_scores(ll):
    attend(ll, "f16", 2, 2, 64, 16, [1, 1], [50, 700], ragged=False, scale=0.5)
    attend(ll, "bf16", 2, 1, 128, 16, [40, 3], [50, 700], scale=0.01)
    attend(ll, "f16", 2, 2, 128, 16, [1, 1], [50, 700], ragged=False, qscale=8.0)      # one key outweighs the rest
    attend(ll, "f16", 2, 2, 128, 16, [40, 40], [50, 700], qscale=8.0)
    attend(ll, "bf16", 2, 2, 128, 16, [1, 40], [50, 700], qscale=2.0 ** -100)
    attend(ll, "bf16", 2, 2, 128, 16, [1, 40], [50, 700], qscale=2.0 ** 100, scale=2.0 ** -103)


def test_zero_queries_average_the_values(ll):
    attend(ll, "f16", 2, 2, 128, 16, [1, 40], [1000, 50], qscale=0.0)


@pytest.mark.parametrize("rows", [1, 40])
def test_nan_in_a_row_stays_in_it(ll, rows):
    lens, page = [300, 300], 16
    table, pages, at = ku.paged(lens, page)
    raw, pool = ku.random_pool(2, 128, pages * page, at, 0)
    q = torch.randn(2 * rows, 2, 128).half()
    q[0, 1, 5] = float("nan")
    r = ll.KV4Rows(ints(lens), ints(table), max_rows=rows)
    cache = ll.KV4Cache(dev(raw), 2, 128, page, pages)
    good = ll.ll_kv4_attention(cache, r, dev(torch.where(q.isnan(), 0, q))).cpu()
    got = ll.ll_kv4_attention(cache, r, dev(q)).cpu()
    assert got[0, 1].isnan().all()
    mask = torch.ones(2 * rows, 2, dtype=torch.bool)
    mask[0, 1] = False
    assert torch.equal(got[mask], good[mask])
    # a NaN held in a value reaches the rows that see it, in its own group of 32
    pool.params[1][1, int(at[1][290 - rows]), 2] = float("nan")
    got = ll.ll_kv4_attention(ll.KV4Cache(dev(raw), 2, 128, page, pages), r, dev(torch.where(q.isnan(), 0, q))).cpu()
    assert got[rows:, 1, 64:96].isnan().all()
    got[rows:, 1, 64:96] = good[rows:, 1, 64:96]
    assert torch.equal(got, good)


def test_rows_behind_the_last_sequence_are_left_alone(ll):
    table, pages, at = ku.paged([40, 50], 16)
    raw, _ = ku.random_pool(2, 64, pages * 16, at, 0)
    for m in ([1, 1], [20, 30]):
        n = sum(m) + 3
        out = torch.full((n, 2, 64), 9.0, dtype=torch.float16, device="cuda:0")
        r = ll.KV4Rows(ints([40, 50]), ints(table), max_rows=max(m), row_start=ints([0, m[0], m[0] + m[1]]))
        ll.ll_kv4_attention(ll.KV4Cache(dev(raw), 2, 64, 16, pages), r, torch.randn(n, 2, 64, device="cuda:0").half(), out=out)
        assert (out[-3:] == 9).all() and (out[:-3] != 9).any(-1).all()


def test_sequences_that_share_pages(ll):
    """Two sequences with the same first pages give the same as with a copy each."""
    raw, _ = ku.random_pool(2, 128, 16 * 16, [np.arange(256)], 0)
    q = torch.randn(2, 2, 128).half()
    cache = ll.KV4Cache(dev(raw), 2, 128, 16, 16)
    both = ll.ll_kv4_attention(cache, ll.KV4Rows(ints([60, 70]), ints([[32, 64, 16, 80, -1], [32, 64, 16, 96, 112]])), dev(q))
    for b in range(2):
        one = ll.ll_kv4_attention(cache, ll.KV4Rows(ints([[60, 70][b]]), ints([[[32, 64, 16, 80, -1], [32, 64, 16, 96, 112]][b]])), dev(q[b:b + 1]))
        assert torch.equal(one[0], both[b])


@pytest.mark.parametrize("kv_heads,pages,page", [(1, 1 << 14, 1 << 12), (40, 1 << 9, 1 << 12)])
def test_offsets_beyond_32_bits(ll, kv_heads, pages, page):
    """The last pool rows: their bytes lie 4 GiB behind a head's first, or the head itself does."""
    rows_, hd = pages * page, 128
    nbytes = ll.ll_kv4_pool_bytes(kv_heads, hd, page, pages)
    assert nbytes > 10 << 29
    pool = torch.zeros(nbytes, dtype=torch.uint8, device="cuda:0")
    cache = ll.KV4Cache(pool, kv_heads, hd, page, pages)
    g = torch.Generator().manual_seed(0)
    k, v = (torch.randn(50, kv_heads, hd, generator=g).half() for _ in range(2))
    r = ll.KV4Rows(ints([50]), ints([[(pages - 1) * page]]), max_rows=50)
    ll.ll_kv4_write(cache, r, dev(k), dev(v))
    held = [ku.values(*ku.quantise(x)) for x in (k, v)]
    back = ll.ll_kv4_read(cache, r, n_rows=50, dtype=torch.float16)
    for x, y in zip(back, held):
        assert ((x.cpu().double() - y).abs() <= 2.0 ** -10 * y.abs() + 2.0 ** -25).all()
    q = torch.randn(50, kv_heads, hd, generator=g).half()
    for m, rr in ((50, r), (1, ll.KV4Rows(ints([50]), ints([[(pages - 1) * page]])))):
        out = ll.ll_kv4_attention(cache, rr, dev(q[:m]))
        want, tol = ku.attention(q[:m].double(), held[0].transpose(0, 1), held[1].transpose(0, 1),
                                 [50] if m == 1 else range(1, 51), hd ** -0.5)
        ku.check_attention(out, want, tol, "at the end of a large pool")
    assert not pool[:4096].any()


# ---- streams, graphs, workspaces ----

def test_on_another_stream(ll):
    table, pages, at = ku.paged([700, 50], 16)
    raw, _ = ku.random_pool(2, 128, pages * 16, at, 0)
    cache, r = ll.KV4Cache(dev(raw), 2, 128, 16, pages), ll.KV4Rows(ints([700, 50]), ints(table))
    q = torch.randn(2, 4, 128, device="cuda:0").half()
    want = ll.ll_kv4_attention(cache, r, q)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = ll.ll_kv4_attention(cache, r, q, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    with torch.cuda.stream(s):
        got = ll.ll_kv4_attention(cache, r, q)
        k, v = ll.ll_kv4_read(cache, r, n_rows=2, dtype=torch.float16)
    s.synchronize()
    assert torch.equal(got, want)
    assert torch.equal(k, ll.ll_kv4_read(cache, r, n_rows=2, dtype=torch.float16)[0])


@pytest.mark.parametrize("rows", [1, 24])
def test_captured_calls_follow_what_lies_in_memory(ll, rows):
    """A step captured once: every replay writes its new rows and attends, at lengths that grow between the replays; two
    graphs take turns on one workspace."""
    hd, kv, heads, page = 128, 2, 8, 16
    lens, top = [40, 900, 7 + rows], 1000
    table, pages, at = ku.paged([top] * 3, page)
    raw, _ = ku.random_pool(kv, hd, pages * page, [a[:n] for a, n in zip(at, lens)], 0)
    pool, eager_pool = dev(raw.clone()), dev(raw.clone())
    dl, dt = ints(lens), ints(table)
    x = torch.randn(3 * rows, heads + 2 * kv, hd, device="cuda:0").half()
    q, k, v = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
    cache, other = ll.KV4Cache(pool, kv, hd, page, pages), ll.KV4Cache(eager_pool, kv, hd, page, pages)
    r = ll.KV4Rows(dl, dt, max_rows=rows)
    ws = torch.empty(max(1, ll.ll_kv4_attention_workspace_bytes(cache, r, heads, 3 * rows)), dtype=torch.uint8, device="cuda:0")
    outs, graphs = [torch.empty_like(q) for _ in range(2)], []
    ll.ll_kv4_attention(other, r, q, k=k, v=v)          # loads the kernels
    eager_pool.copy_(dev(raw))
    for o in outs:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            ll.ll_kv4_attention(cache, r, q, k=k, v=v, out=o, workspace=ws)
        graphs.append(gr)
    for step in range(6):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(step)).half())
        dl += rows
        graphs[step % 2].replay()
        torch.cuda.synchronize()
        want = ll.ll_kv4_attention(other, r, q, k=k, v=v)
        assert torch.equal(outs[step % 2], want), step
        assert torch.equal(pool, eager_pool)


def test_the_same_call_gives_the_same_bits(ll):
    table, pages, at = ku.paged([5000, 300, 40], 16)
    raw, _ = ku.random_pool(2, 128, pages * 16, at, 0)
    cache, r = ll.KV4Cache(dev(raw), 2, 128, 16, pages), ll.KV4Rows(ints([5000, 300, 40]), ints(table))
    q = torch.randn(3, 8, 128, device="cuda:0").half()
    first = ll.ll_kv4_attention(cache, r, q)
    for _ in range(5):
        assert torch.equal(ll.ll_kv4_attention(cache, r, q), first)


# ---- refusals ----

def test_refusals(ll):
    table, pages, at = ku.paged([40], 16)
    raw, _ = ku.random_pool(2, 64, pages * 16, at, 0)
    pool = dev(raw)
    cache, r = ll.KV4Cache(pool, 2, 64, 16, pages), ll.KV4Rows(ints([40]), ints(table))
    q = torch.randn(1, 4, 64, device="cuda:0").half()
    before = pool.clone()

    def refused(code, call):
        with pytest.raises(ll.LLError) as e:
            call()
        assert e.value.code == code
    refused(ll.LL_E_BAD_CONFIG, lambda: ll.ll_kv4_attention(cache, r, q[:, :3]))
    refused(ll.LL_E_BAD_ARG, lambda: ll.ll_kv4_attention(cache, r, q, scale=float("nan")))
    refused(ll.LL_E_BAD_ARG, lambda: ll.ll_kv4_attention(cache, r, q, scale=-1.0))
    refused(ll.LL_E_BAD_ARG, lambda: ll.ll_kv4_attention(cache, r, q, k=q[:, :2]))
    refused(ll.LL_E_BAD_ARG, lambda: ll.ll_kv4_attention(cache, r, q.expand(2, 4, 64)))       # two rows, one sequence of one
    refused(ll.LL_E_BAD_ARG, lambda: ll.ll_kv4_attention(cache, r, q, out=q[:, :1].expand(1, 4, 64)))
    refused(ll.LL_E_WORKSPACE, lambda: ll.ll_kv4_write(ll.KV4Cache(pool, 2, 64, 16, pages + 1), r, q[:, :2], q[:, :2]))
    refused(ll.LL_E_WORKSPACE, lambda: ll.ll_kv4_write(ll.KV4Cache(pool[16:], 1, 64, 16, pages), r, q[:, :1], q[:, :1]))
    for bad in (lambda: ll.ll_kv4_attention(cache, r, q.float()), lambda: ll.ll_kv4_write(cache, r, q, q),
                lambda: ll.ll_kv4_write(cache, r, q[:, :2], q[:, :2].bfloat16()),
                lambda: ll.ll_kv4_attention(cache, r, q, out=q.bfloat16()),
                lambda: ll.KV4Rows(ints([40]).long(), ints(table)), lambda: ll.KV4Rows(ints([40, 1]), ints(table)),
                lambda: ll.ll_kv4_attention(cache, r, q.transpose(1, 2))):
        with pytest.raises(ValueError):
            bad()
    assert torch.equal(pool, before)


def test_empty_calls(ll):
    pool = torch.zeros(ll.ll_kv4_pool_bytes(2, 64, 16, 2), dtype=torch.uint8, device="cuda:0")
    cache = ll.KV4Cache(pool, 2, 64, 16, 2)
    r = ll.KV4Rows(ints(np.zeros(0)), ints(np.zeros((0, 3))))
    none = torch.empty(0, 2, 64, dtype=torch.float16, device="cuda:0")
    ll.ll_kv4_write(cache, r, none, none)
    assert ll.ll_kv4_attention(cache, r, none).shape == (0, 2, 64)
