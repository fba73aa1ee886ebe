"""A key/value cache held in 4 bits: the calls that write it, read it back and attend over it, and what they compute.

Where ``own`` is false, ``run`` computes the operators with elementary torch operations; where it is true, it calls the
library.  Both take the same cache bytes.

Format, for every group of 32 consecutive elements of one head's key or value row:  value = mid + s (c - 8)
    t = max - min,  s = smallest binary16 number of at most 8 significant bits with 15 s >= t,  mid = binary16(min + 8 s),
    c = 8 + clamp(round((x - mid) / s), -8, 7), rounded half to even, 8 where s = 0.
The pool of a layer holds [K codes][V codes][K parameters][V parameters], each region padded to 256 bytes: codes are
[kv head][pool row][head_dim / 2] bytes (element 2 j in the low half of byte j, 2 j + 1 in the high one), parameters
[kv head][pool row][head_dim / 32][s, mid].  page_table[b][i] is the first pool row of sequence b's page i.
"""
import math

import numpy as np
import torch

own = False

GROUP = 32
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # one new token of the two-layer toy decoder: nothing but latency
        dict(name="step toy 1x41", kind="step", dtype="f16", heads=4, kv_heads=4, head_dim=64, page=16, seqs=1, rows=1,
             ragged=0, ctx_from=40, ctx_to=40),
        # a batched step at the 7B head layout, prompts and answers of mixed length
        dict(name="step 16x10..560", kind="step", dtype="f16", heads=32, kv_heads=32, head_dim=128, page=16, seqs=16, rows=1,
             ragged=0, ctx_from=9, ctx_to=559),
        # the fullest batch, two thousand positions each
        dict(name="step 32x1500..2500", kind="step", dtype="f16", heads=32, kv_heads=32, head_dim=128, page=32, seqs=32, rows=1,
             ragged=0, ctx_from=1500, ctx_to=2500),
        # few long documents, key heads shared by four query heads: the work has to be split along the keys
        dict(name="step 4x30000 shared heads", kind="step", dtype="bf16", heads=32, kv_heads=8, head_dim=128, page=64, seqs=4, rows=1,
             ragged=0, ctx_from=30000, ctx_to=33001),
        # attention of a whole 500-token prompt
        dict(name="prompt 500", kind="attention", dtype="f16", heads=32, kv_heads=32, head_dim=128, page=16, seqs=1, rows=500,
             ragged=0, ctx_from=0, ctx_to=0),
        # prompts of several lengths behind cached positions, in one call
        dict(name="prompts 6x1..700 shared heads", kind="attention", dtype="bf16", heads=32, kv_heads=8, head_dim=128, page=48, seqs=6, rows=700,
             ragged=1, ctx_from=0, ctx_to=2001),
        # the last chunk of an 8 K prompt
        dict(name="chunk 1024 behind 7169", kind="attention", dtype="f16", heads=32, kv_heads=32, head_dim=128, page=128, seqs=1, rows=1024,
             ragged=0, ctx_from=7169, ctx_to=7169),
        # one row of each of 16 sequences into the cache and back
        dict(name="write 16x1", kind="write", dtype="f16", heads=32, kv_heads=32, head_dim=128, page=16, seqs=16, rows=1,
             ragged=0, ctx_from=9, ctx_to=559),
        # a 500-token prompt's rows
        dict(name="write 500", kind="write", dtype="f16", heads=32, kv_heads=32, head_dim=128, page=16, seqs=1, rows=500,
             ragged=0, ctx_from=0, ctx_to=0),
        # long prompts out of a fused projection's output
        dict(name="write 4x1..8190", kind="write", dtype="bf16", heads=32, kv_heads=8, head_dim=128, page=64, seqs=4, rows=8190,
             ragged=1, ctx_from=0, ctx_to=0),
        # a sequence of the toy decoder read back
        dict(name="read toy 63", kind="read", dtype="f16", heads=4, kv_heads=4, head_dim=64, page=16, seqs=1, rows=63,
             ragged=0, ctx_from=0, ctx_to=0),
        # a whole batch read back
        dict(name="read 32x1..1000", kind="read", dtype="bf16", heads=32, kv_heads=32, head_dim=128, page=32, seqs=32, rows=1000,
             ragged=1, ctx_from=0, ctx_to=0),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """Any head layout, page size and type; lengths spread over their logarithm, no dearer than the dearest listed case."""
    kind = rng.choice(["step", "step", "attention", "attention", "write", "read"])
    head_dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 5, 8, 16, 32])
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 7, 8])
    heads = heads if heads <= 64 else kv_heads
    case = dict(kind=kind, dtype=rng.choice(["f16", "bf16"]), heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                page=rng.choice([1, 7, 16, 16, 24, 32, 64, 128, 256]))
    seqs = _log(rng, 1, 64)
    if kind == "step":
        most = max(16, min(32768, 2000000 // (seqs * kv_heads)))
        top = _log(rng, 8, most)
        ctx, rows, ragged = [rng.randint(0, top), top], 1, 0
    elif kind == "attention":
        seqs = _log(rng, 1, 8)
        rows = _log(rng, 2, max(2, 4096 // (seqs * max(1, heads // 8))))
        top = _log(rng, 1, max(2, min(8192, 150000000 // (seqs * heads * rows))))
        ctx, ragged = [rng.randint(0, top), top], rng.randint(0, 1)
    else:
        rows = _log(rng, 1, max(2, 500000 // (seqs * kv_heads)))
        ctx, ragged = [0, 0] if kind == "read" else [0, _log(rng, 1, 500)], rng.randint(0, 1)
    return dict(case, seqs=seqs, rows=rows, ragged=ragged, ctx_from=ctx[0], ctx_to=ctx[1])


def _spread(low, high, n):
    """n whole numbers from low to high, evenly spread."""
    return [low + ((high - low) * i + (n - 1) // 2) // max(1, n - 1) for i in range(n)] if n > 1 else [high]


def _lengths(case):
    """(rows, cached positions in front of them) of every sequence, before they are shuffled."""
    m = _spread(1, case["rows"], case["seqs"]) if case["ragged"] else [case["rows"]] * case["seqs"]
    return m, _spread(case["ctx_from"], case["ctx_to"], case["seqs"])


def _regions(case, pool_rows):
    """Byte offsets of the pool's four regions, and its size."""
    pad = lambda n: (n + 255) // 256 * 256  # noqa: E731
    codes = pad(case["kv_heads"] * pool_rows * case["head_dim"] // 2)
    params = pad(case["kv_heads"] * pool_rows * case["head_dim"] // GROUP * 4)
    return 0, codes, 2 * codes, 2 * codes + params, 2 * codes + 2 * params


def _shuffled(values, n, seed):
    order = np.random.RandomState(seed).permutation(n)
    return [values[i] for i in order]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, hd, kv = DTYPES[case["dtype"]], case["head_dim"], case["kv_heads"]
    m, ctx = _lengths(case)
    ctx = _shuffled(ctx, case["seqs"], seed % 65521)
    m = _shuffled(m, case["seqs"], seed % 65521 + 1)
    lens = np.array(ctx) + np.array(m)
    start = np.concatenate([[0], np.cumsum(m)])
    pages = [-(-int(n) // case["page"]) for n in lens]
    stride = max(pages) + 1
    total = sum(pages) + 2
    free = np.random.RandomState(seed % 65521 + 2).permutation(total)          # pages of a sequence lie anywhere in the pool
    table = np.full((case["seqs"], stride), 0, dtype=np.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = free[at:at + n] * case["page"]
        at += n
    pool_rows = total * case["page"]
    off = _regions(case, pool_rows)
    pool = torch.empty(off[4], dtype=torch.uint8, device="cuda")
    # codes as a normal variable's lie: the sum of two numbers of three bits and one of one bit, in both halves of a byte
    shape = (2 * off[1],)
    half = lambda bits: torch.randint(0, 256, shape, dtype=torch.uint8, device="cuda", generator=g) & bits  # noqa: E731
    pool[:2 * off[1]] = half(0x77) + half(0x77) + half(0x11)
    n_groups = kv * pool_rows * hd // GROUP
    params = pool[off[2]:off[4]].view(torch.float16).view(2, -1)
    for which in range(2):
        s = 0.18 + 0.18 * torch.rand(n_groups, device="cuda", generator=g)
        s = (s * 512).round() / 512                                             # at most 8 significant bits
        mid = 0.1 * torch.randn(n_groups, device="cuda", generator=g)
        if which == 0:                                                          # keys have channels that are always off
            mid = (mid.view(kv, pool_rows, -1) + torch.randn(kv, 1, hd // GROUP, device="cuda", generator=g)).reshape(-1)
        params[which, :2 * n_groups] = torch.stack([s, mid], -1).reshape(-1).to(torch.float16)
    state = dict(case=case, pool=pool, pool_rows=pool_rows, pages=total,
                 lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
                 start=torch.tensor(start, dtype=torch.int32, device="cuda") if case["ragged"] else None,
                 table=torch.tensor(table, device="cuda"), n_rows=int(start[-1]), max_len=int(lens.max()))
    # rows that no sequence has written hold what the memory held before: here NaN
    used = torch.zeros(pool_rows, dtype=torch.bool, device="cuda")
    where, inside = _positions(state, state["max_len"])
    used[where[inside]] = True
    for which in range(2):
        p = params[which, :2 * n_groups].view(kv, pool_rows, -1)
        p[:, ~used] = float("nan")
    # q, k, v: the output of one projection, rows of all heads side by side
    both = case["heads"] + 2 * kv
    x = torch.randn(state["n_rows"], both, hd, device="cuda", generator=g)
    x[:, case["heads"]:case["heads"] + kv] += torch.randn(1, kv, hd, device="cuda", generator=g)
    x = x.to(dt)
    state["q"], state["k"], state["v"] = x[:, :case["heads"]], x[:, case["heads"]:case["heads"] + kv], x[:, case["heads"] + kv:]
    return state


def work(case):
    m, ctx = _lengths(case)
    row = case["kv_heads"] * case["head_dim"]
    held = row // 2 + row // GROUP * 4                                          # bytes of one position's keys or values
    rows, keys = sum(m), sum(m) + sum(ctx)
    if case["kind"] == "write":
        return {"bytes": 2 * rows * (2 * row + held) + 2 * rows * (2 * row + held), "flops": 2 * rows * row * 8}
    if case["kind"] == "read":
        return {"bytes": 2 * rows * (2 * row + held), "flops": 2 * rows * row * 2}
    # the lists are shuffled: a row sees its sequence's cached positions in the mean, and the rows up to itself
    seen = sum(n * sum(ctx) / len(ctx) + n * (n + 1) / 2 for n in m)
    bytes_ = 2 * keys * held + 2 * rows * case["heads"] * case["head_dim"] * 2
    if case["kind"] == "step":
        bytes_ += 2 * rows * 2 * row * 2                                        # the new rows in, and their values back
    return {"bytes": bytes_, "flops": 4 * case["heads"] * case["head_dim"] * seen}


# ---- plain form ----

def _positions(state, most):
    """[sequence][position] -> pool row, and which positions exist."""
    pos = torch.arange(most, device="cuda")
    page = state["case"]["page"]
    row = state["table"][:, pos // page].long() + (pos % page)
    return row, pos[None, :] < state["lens"][:, None]


def _rows(state):
    """Sequence and position of every row of the call."""
    rows = torch.arange(state["n_rows"], device="cuda")
    if state["start"] is None:
        m = state["case"]["rows"]
        b = rows // m
        return b, state["lens"][b].long() - m + rows % m
    start = state["start"].long()
    b = torch.searchsorted(start, rows, right=True) - 1
    return b, state["lens"][b].long() - (start[b + 1] - rows)


def _held(state, which, rows):
    """Values of the keys (0) or values (1) in the given pool rows: [kv head, *rows.shape, head_dim]."""
    case, off = state["case"], _regions(state["case"], state["pool_rows"])
    kv, hd = case["kv_heads"], case["head_dim"]
    n = kv * state["pool_rows"]
    codes = state["pool"][off[which]:off[which] + n * hd // 2].view(kv, state["pool_rows"], hd // 2)[:, rows]
    params = state["pool"][off[2 + which]:off[2 + which] + n * hd // GROUP * 4].view(torch.float16)
    params = params.view(kv, state["pool_rows"], hd // GROUP, 2)[:, rows].float()
    c = torch.stack([codes & 15, codes >> 4], -1).float().flatten(-2).unflatten(-1, (hd // GROUP, GROUP))
    return (params[..., 1:] + params[..., :1] * (c - 8)).flatten(-2)


def _store(state, which, x, rows):
    """Quantises x [row, kv head, head_dim] into the given pool rows."""
    case, off = state["case"], _regions(state["case"], state["pool_rows"])
    kv, hd = case["kv_heads"], case["head_dim"]
    n = kv * state["pool_rows"]
    x = x.double().unflatten(-1, (hd // GROUP, GROUP))                           # borders between two codes decide in 64 bits
    low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    t = (high - low) / 15
    step = torch.where(t > 0, t / torch.frexp(t)[0] / 256, 1.0).clamp_min(2.0 ** -24)   # t / its mantissa: a power of two
    s = torch.ceil(t / step) * step
    mid = (low + 8 * s).to(torch.float16).double()
    c = 8 + torch.where(s > 0, (x - mid) / s, 0.0).round().clamp(-8, 7)
    c = c.to(torch.uint8).flatten(-2)
    codes = state["pool"][off[which]:off[which] + n * hd // 2].view(kv, state["pool_rows"], hd // 2)
    codes[:, rows] = (c[..., 0::2] | c[..., 1::2] << 4).transpose(0, 1)
    params = state["pool"][off[2 + which]:off[2 + which] + n * hd // GROUP * 4].view(torch.float16)
    params.view(kv, state["pool_rows"], hd // GROUP, 2)[:, rows] = torch.cat([s, mid], -1).to(torch.float16).transpose(0, 1)


def _plain_read(state, b, pos):
    rows = state["table"][b, pos // state["case"]["page"]].long() + pos % state["case"]["page"]
    dt = DTYPES[state["case"]["dtype"]]
    return tuple(_held(state, which, rows).transpose(0, 1).to(dt).contiguous() for which in range(2))


def _plain_write(state, b, pos):
    rows = state["table"][b, pos // state["case"]["page"]].long() + pos % state["case"]["page"]
    _store(state, 0, state["k"], rows)
    _store(state, 1, state["v"], rows)


def _plain_attention(state, b, pos):
    """Every sequence's rows and keys padded to the longest; what a row does not see is masked."""
    case, n, m = state["case"], state["case"]["seqs"], state["case"]["rows"]
    kv, hd, share = case["kv_heads"], case["head_dim"], case["heads"] // case["kv_heads"]
    first = torch.arange(n, device="cuda") * m if state["start"] is None else state["start"][:-1].long()
    j = torch.arange(state["n_rows"], device="cuda") - first[b]
    q = torch.zeros(n, m, kv, share, hd, device="cuda")
    q[b, j] = state["q"].float().unflatten(1, (kv, share))
    last = torch.full((n, m), -1, dtype=torch.long, device="cuda")
    last[b, j] = pos
    where, inside = _positions(state, state["max_len"])
    k, v = (torch.where(inside[None, :, :, None], _held(state, which, where), 0.0).transpose(0, 1) for which in range(2))
    q = q.permute(0, 2, 1, 3, 4).reshape(n, kv, m * share, hd)
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(hd)
    scores = scores.view(n, kv, m, share, -1)
    seen = torch.arange(state["max_len"], device="cuda")[None, None] <= last[:, :, None]
    scores.masked_fill_(~seen[:, None, :, None], float("-inf"))
    p = scores - scores.amax(-1, keepdim=True).clamp_min(-3e38)
    p = p.exp_()
    p = p / p.sum(-1, keepdim=True).clamp_min(1e-37)
    out = torch.matmul(p.view(n, kv, m * share, -1), v.contiguous()).view(n, kv, m, share, hd)
    return out.permute(0, 2, 1, 3, 4)[b, j].flatten(1, 2).to(DTYPES[case["dtype"]])


# ---- the library's calls ----

def _own(state):
    from paper_2604_23467_amd import binding as ll
    case = state["case"]
    cache = ll.KV4Cache(state["pool"], case["kv_heads"], case["head_dim"], case["page"], state["pages"])
    rows = ll.KV4Rows(state["lens"], state["table"], max_rows=case["rows"], row_start=state["start"])
    if case["kind"] == "attention":
        return ll.ll_kv4_attention(cache, rows, state["q"])
    if case["kind"] == "step":
        out = ll.ll_kv4_attention(cache, rows, state["q"], k=state["k"], v=state["v"])
        return (out,) + ll.ll_kv4_read(cache, rows, n_rows=state["n_rows"], dtype=state["q"].dtype)
    if case["kind"] == "write":
        ll.ll_kv4_write(cache, rows, state["k"], state["v"])
    return ll.ll_kv4_read(cache, rows, n_rows=state["n_rows"], dtype=state["q"].dtype)


def run(state):
    """attention: the rows' outputs.  step: the new keys and values are written, then attended with everything before them;
    outputs and what the cache holds of the new rows.  write: what the cache then holds of the rows.  read: that alone."""
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    b, pos = _rows(state)
    if kind in ("step", "write"):
        _plain_write(state, b, pos)
    if kind == "attention":
        return _plain_attention(state, b, pos)
    held = _plain_read(state, b, pos)
    return (_plain_attention(state, b, pos),) + held if kind == "step" else held


# ---- the definition in 64 bits ----

def _exact_values(x):
    """What the format holds of x [..., head_dim], by the definition."""
    x = x.double()
    y = x.reshape(*x.shape[:-1], -1, GROUP)
    low = y.min(-1, keepdim=True).values
    span = y.max(-1, keepdim=True).values - low
    # 8 significant bits, binary16's smallest step at least
    power = torch.clamp(torch.floor(torch.log2(torch.clamp(span / 15, min=2.0 ** -60))) - 7, min=-24)
    unit = (power.long() + 1023 << 52).view(torch.float64)                       # 2 ** power by its bits
    s = unit * torch.ceil(span / (15 * unit))
    mid = (low + 8 * s).half().double()
    c = torch.clamp(torch.round((y - mid) / torch.where(s == 0, 1.0, s)), -8, 7)
    return (mid + s * c).reshape(x.shape)


def exact(case, seed):
    st = prepare(case, seed)
    kv, hd, share = case["kv_heads"], case["head_dim"], case["heads"] // case["kv_heads"]
    lens, table = st["lens"].tolist(), st["table"].long()
    start = st["start"].tolist() if st["start"] is not None else [case["rows"] * b for b in range(case["seqs"] + 1)]
    seen = sum((start[b + 1] - start[b]) * lens[b] for b in range(case["seqs"]))
    if case["kind"] in ("step", "attention") and seen * case["heads"] * hd * 4 > 4e12:
        return None
    codes, params = [], []
    at = 0
    for size, to in ((hd // 2, codes), (hd // GROUP * 4, params)):
        for _ in range(2):
            n = kv * st["pool_rows"] * size
            to.append(st["pool"][at:at + n].view(kv, st["pool_rows"], size))
            at += (n + 255) // 256 * 256

    def values(b, which, low, high):
        """[kv head, positions low .. high - 1, head_dim] of sequence b"""
        u = torch.arange(low, high, device="cuda")
        r = table[b][u // case["page"]] + u % case["page"]
        byte = codes[which][:, r]
        c = torch.empty(kv, high - low, hd, dtype=torch.float64, device="cuda")
        c[..., 0::2], c[..., 1::2] = (byte % 16).double(), (byte // 16).double()
        p = params[which][:, r].contiguous().view(torch.float16).double().reshape(kv, high - low, hd // GROUP, 2)
        return (p[..., 1].repeat_interleave(GROUP, -1) + p[..., 0].repeat_interleave(GROUP, -1) * (c - 8))

    new = [_exact_values(st["k"]), _exact_values(st["v"])]                       # [row, kv head, head_dim]
    if case["kind"] == "write":
        return tuple(new)
    held, outs = [[], []], []
    for b in range(case["seqs"]):
        m, n = start[b + 1] - start[b], lens[b]
        if case["kind"] == "read":
            for which in range(2):
                held[which].append(values(b, which, n - m, n).transpose(0, 1))
            continue
        k, v = values(b, 0, 0, n), values(b, 1, 0, n)
        if case["kind"] == "step":
            k[:, n - m:], v[:, n - m:] = new[0][start[b]:start[b + 1]].transpose(0, 1), new[1][start[b]:start[b + 1]].transpose(0, 1)
        q = st["q"][start[b]:start[b + 1]].double()
        out = torch.empty(m, case["heads"], hd, dtype=torch.float64, device="cuda")
        for h in range(kv):
            for j in range(0, m, 512):
                e = min(m, j + 512)
                top = n - m + e                                                  # keys that the last of these rows sees
                x = q[j:e, h * share:(h + 1) * share].reshape(-1, hd) @ k[h, :top].T / hd ** 0.5
                lim = (n - m + torch.arange(j, e, device="cuda")).repeat_interleave(share)
                x[torch.arange(top, device="cuda")[None] > lim[:, None]] = float("-inf")
                out[j:e, h * share:(h + 1) * share] = (torch.softmax(x, -1) @ v[h, :top]).reshape(e - j, share, hd)
        outs.append(out)
    if case["kind"] == "read":
        return tuple(torch.cat(x) for x in held)
    return (torch.cat(outs),) + tuple(new) if case["kind"] == "step" else torch.cat(outs)
