"""Cases of serving from a cache in pages: the step from the projections to the cache (norm of every query and key head,
rotation, cast, write), attention of a ragged batch of new tokens over a contiguous or paged cache with a sliding window and
first tokens that stay visible, and the bookkeeping and copying of pages.

A pool of pages is a cache whose first index is the page: planes [pages, heads, page tokens, bytes].  A row holds 128 slots in
block floating point: blocks of ``block`` slots share an exponent byte E + 127, a slot holds M + 2^(bits-1) in ``bits`` bits of a
little-endian stream, its value is M 2^(E-(bits-2)); slot j of a head holds channel perm[j].
"""
import math

import numpy as np
import torch

own = False

D = 128
PLANES = ("k_mant", "k_exp", "v_mant", "v_exp")


# ---------------------------------------------------------------------------------------------------- the cases
def _case(name, op, batch, kv_heads, group, seq, bits, block, dtype, **more):
    c = {"name": name, "op": op, "batch": batch, "kv_heads": kv_heads, "group": group, "seq": seq, "bits": bits,
         "block": block, "dtype": dtype, "page": 0, "new": 1, "ragged": False, "window": 0, "sink": 0, "half": False,
         "branches": 0, "fill": 0}
    c.update(more)
    return c


def listed():
    return [
        # one user's next token on its way into the cache: the smallest call, all latency
        _case("write token b1 gqa", "write", 1, 8, 4, 5000, 4, 32, "bf16", page=16),
        # the next tokens of a batch of users, 8-bit rows
        _case("write tokens b64 8bit", "write", 64, 32, 1, 2048, 8, 32, "bf16", page=64, half=True),
        # the prompts of a ragged batch
        _case("write prompts b4 gqa", "write", 4, 8, 4, 8192, 4, 32, "bf16", new=8192, ragged=True, half=True),
        # one user's next token under a sliding window whose first tokens stay visible
        _case("attend token b1 window", "attend", 1, 32, 1, 4096, 4, 32, "bf16", page=16, window=1000, sink=4),
        # the next tokens of a batch of users over long histories
        _case("attend tokens b16 h32", "attend", 16, 32, 1, 8192, 4, 32, "bf16", page=64),
        # grouped heads, ragged histories, pages shorter than a tile
        _case("attend tokens b8 gqa", "attend", 8, 8, 4, 32768, 4, 32, "bf16", page=32, ragged=True),
        # a few fp32 tokens each over 6-bit rows, window and sinks: full accuracy
        _case("attend f32 6bit", "attend", 3, 2, 3, 1003, 6, 16, "f32", page=16, new=5, ragged=True, window=300, sink=3),
        # a whole prompt read back from the cache it has just been written to
        _case("attend prompt b1 h32", "attend", 1, 32, 1, 8192, 4, 32, "bf16", new=8192),
        # chunks of long prompts under a sliding window, 8-bit rows
        _case("attend chunks b4 window", "attend", 4, 8, 4, 16384, 8, 32, "bf16", page=128, new=2048, window=4096, sink=16),
        # a batch in which some users prefill a chunk while others decode a token
        _case("attend mixed b16 gqa", "attend", 16, 8, 4, 8192, 4, 32, "bf16", page=64, new=512, ragged=True),
        # branches of running sequences dropped and forked anew, the page each of them writes next made its own
        _case("branch b8 x 4", "branch", 8, 8, 1, 8191, 4, 32, "bf16", page=64, branches=4, new=3),
        # the pages in use of a large pool packed into another
        _case("pack 16384 pages", "pack", 64, 8, 1, 16384, 4, 32, "bf16", page=64, fill=16384),
        ]


def draw(rng):
    """Any operator over its range, every format."""
    op = rng.choice(["write", "write", "attend", "attend", "attend", "attend", "branch", "pack"])
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))
    bits, block = rng.choice([4, 4, 4, 6, 8]), rng.choice([16, 32, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    page = rng.choice([0, 16, 16, 32, 64, 64, 128, 256])
    batch, kv_heads, group = log(1, 16), rng.choice([1, 2, 3, 4, 8, 8, 16, 32]), rng.choice([1, 1, 2, 3, 4, 4, 8])
    if op == "write":
        batch = log(1, 64)
        new = rng.choice([1, 1, log(1, 8192)])
        new = max(1, min(new, (1 << 20) // (batch * kv_heads * (group + 2))))
        c = _case("", op, batch, kv_heads, group, new + log(1, 2048), bits, block, dtype, page=page, new=new,
                  ragged=rng.random() < 0.5, half=rng.random() < 0.5)
    elif op == "attend":
        seq = log(1, min(32768, (1 << 21) // (batch * kv_heads)))
        new = rng.choice([1, 1, log(1, 8), log(1, 2048)])
        cost = (1 << 31) if dtype == "bf16" else (1 << 26)          # query heads times new tokens times cached tokens
        new = max(1, min(new, seq, cost // (batch * kv_heads * group * seq)))
        c = _case("", op, batch, kv_heads, group, seq, bits, block, dtype, page=page, new=new, ragged=rng.random() < 0.6)
        if rng.random() < 0.5:
            c["window"], c["sink"] = log(1, seq), rng.choice([0, 4, 17, 130])
    elif op == "branch":
        c = _case("", op, batch, rng.choice([1, 2, 4, 8]), 1, log(1, 8192), bits, block, "bf16", page=max(16, page),
                  branches=rng.randint(1, 8), new=log(1, 200), ragged=rng.random() < 0.7)
    else:
        page = max(16, page)
        fill = log(1, 16384 * 64 // page)
        c = _case("", op, log(1, 64), rng.choice([1, 2, 4, 8]), 1, 16384, bits, block, "bf16", page=page, fill=fill)
    del c["name"]
    return c


def _news(c):
    """New tokens of each sequence."""
    if not c["ragged"]:
        return [c["new"]] * c["batch"]
    if c["op"] == "attend" and c["new"] > 64:            # every other sequence decodes a token
        return [1 if b % 2 else c["new"] - (c["new"] * ((b * 29) % 64)) // 80 for b in range(c["batch"])]
    return [max(1, c["new"] - (c["new"] * ((b * 29) % 64)) // 80) for b in range(c["batch"])]


def _lens(c):
    """Cached tokens of each sequence, the new ones included."""
    if not c["ragged"]:
        return [c["seq"]] * c["batch"]
    return [max(n, c["seq"] - (c["seq"] * ((b * 37) % 64)) // 80) for b, n in enumerate(_news(c))]


def _pairs(c):
    """(cached tokens that any query sees, pairs of a query and a token it sees), of one head, summed over the batch."""
    seen = pairs = 0
    for n, new in zip(_lens(c), _news(c)):
        p = np.arange(n - new, n, dtype=np.int64)
        lo = np.maximum(0, p - c["window"] + 1) if c["window"] else np.zeros_like(p)
        pairs += int((p + 1 - lo + np.minimum(lo, c["sink"] if c["window"] else 0)).sum())
        seen += n - int(lo[0]) + min(int(lo[0]), c["sink"] if c["window"] else 0)
    return seen, pairs


def _unit(c):
    return 2 * (D * c["bits"] // 8 + D // c["block"])


def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    heads = c["kv_heads"] * c["group"]
    if c["op"] == "write":
        t = sum(_news(c))
        return {"bytes": t * (D * es * (2 * heads + 2 * c["kv_heads"]) + c["kv_heads"] * _unit(c)),
                "flops": t * (heads + c["kv_heads"]) * 7 * D}
    if c["op"] == "attend":
        seen, pairs = _pairs(c)
        return {"bytes": seen * c["kv_heads"] * _unit(c) + 2 * sum(_news(c)) * heads * D * es, "flops": 4 * D * heads * pairs}
    page = c["page"] * c["kv_heads"] * _unit(c)
    if c["op"] == "branch":
        # every branch but one of a page that all its owners write gets its own copy of the page its next token goes to
        copies = sum(c["branches"] for n in _lens(c) if n % c["page"])
        return {"bytes": 2 * copies * page + 4 * c["batch"] * (c["branches"] + 1) * _columns(c), "flops": 0}
    used = (c["fill"] + 1) // 2
    return {"bytes": 2 * used * page + 8 * c["fill"] + 8 * used, "flops": 0}


def _columns(c):
    return (c["seq"] + c["new"] + c["page"] - 1) // c["page"]


# ---------------------------------------------------------------------------------------------------- the inputs
def _unit_of(e8, bits):
    """Value of one mantissa unit for each exponent byte."""
    return ((e8.long() + (1023 - 127 - (bits - 2))) << 52).view(torch.float64)


def _cast(x, bits, block):
    """Values [..., D] -> mantissa bytes [..., D * bits / 8], exponent bytes [..., D / block]; rounded in x's type."""
    b = x.reshape(*x.shape[:-1], D // block, block)
    most = b.abs().amax(-1)
    e8 = most.view(torch.int32) >> 23 if x.dtype == torch.float32 else ((most.view(torch.int64) >> 52) - 1023 + 127).clamp_min(0)
    top = (1 << (bits - 1)) - 1
    m = torch.round(b / _unit_of(e8, bits).to(x.dtype)[..., None]).clamp(-top, top)
    f = (m.to(torch.int32) + (1 << (bits - 1))).reshape(x.shape)
    if bits == 8:
        r = f
    elif bits == 4:
        r = f[..., 0::2] | (f[..., 1::2] << 4)
    else:
        w = f[..., 0::4] | (f[..., 1::4] << 6) | (f[..., 2::4] << 12) | (f[..., 3::4] << 18)
        r = torch.stack((w & 255, (w >> 8) & 255, w >> 16), -1).flatten(-2)
    return r.to(torch.uint8), e8.to(torch.uint8)


def _history(s, c, g, pages, rows, dev):
    """Planes of a cache or pool with a history in them: normal values, some key channels loud and sorted together."""
    H = c["kv_heads"]
    planes = {k: [] for k in PLANES}
    step = max(1, (1 << 24) // (H * rows * D))
    for i in range(0, pages, step):
        n = min(step, pages - i)
        for which in ("k", "v"):
            x = torch.randn(n, H, rows, D, generator=g, device=dev)
            if which == "k":
                x *= s["loud"].gather(-1, s["perm"].long())[:, None]
            m, e = _cast(x, c["bits"], c["block"])
            planes[which + "_mant"].append(m)
            planes[which + "_exp"].append(e)
    for k in PLANES:
        s[k] = torch.cat(planes[k]).contiguous()


def prepare(case, seed):
    c = case
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    B, H, G, P = c["batch"], c["kv_heads"], c["group"], c["page"]
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(np.array(x, dtype=np.int32))).to(dev)
    s = {"case": c}
    # a few loud key channels per head, found by the calibration as an order of the channels
    loud = np.ones((H, D), np.float32)
    for h in range(H):
        loud[h, rng.permutation(D)[:6]] = np.exp(rng.normal(1.5, 0.4, 6))
    s["loud"] = torch.from_numpy(loud).to(dev)
    s["perm"] = i32(np.argsort(loud + 0.01 * rng.random((H, D)), axis=-1, kind="stable"))
    if c["op"] in ("write", "attend"):
        news, lens = _news(c), _lens(c)
        s["starts"], s["lens"] = i32(np.concatenate([[0], np.cumsum(news)])), i32(lens)
        T = sum(news)
        if P:
            cols = (max(lens) + P - 1) // P
            # what the call touches has pages: a write those of its new tokens, attention all of them
            need = [[i for i in range((n + P - 1) // P) if c["op"] == "attend" or i >= (n - m) // P] for n, m in zip(lens, news)]
            pages = sum(len(x) for x in need)
            order, table, at = rng.permutation(pages), np.full((B, cols), -1, np.int32), 0
            for b, x in enumerate(need):
                table[b, x] = order[at:at + len(x)]
                at += len(x)
            s["table"] = i32(table)
            _history(s, c, g, pages, P, dev)
        else:
            _history(s, c, g, B, (max(lens) + 15) // 16 * 16, dev)
        if c["op"] == "attend":
            s["q"] = torch.randn(T, H * G, D, generator=g, device=dev).to(dt)
        else:
            # the projections' output, queries, keys and values of a token side by side
            x = torch.randn(T, H * (G + 2), D, generator=g, device=dev)
            x[:, H * G:H * (G + 1)] *= s["loud"]
            s["qkv"] = x.to(dt)
            s["q_weight"] = 1.0 + 0.2 * torch.randn(D, generator=g, device=dev)
            s["k_weight"] = 1.0 + 0.2 * torch.randn(D, generator=g, device=dev)
            s["theta"] = 10000.0 ** (-2.0 * torch.arange(D // 2, dtype=torch.float64, device=dev) / D)
            s["q_out"] = torch.empty(T, H * G, D, dtype=dt, device=dev)
    elif c["op"] == "branch":
        n, cols = B * (c["branches"] + 1), _columns(c)
        lens, table, at = np.zeros(n, np.int32), np.full((n, cols), -1, np.int32), 0
        pages = sum((x + P - 1) // P for x in _lens(c)) + B * (c["branches"] + 1) * ((c["new"] + P - 1) // P + 1)
        order = rng.permutation(pages)
        for b, x in enumerate(_lens(c)):
            k = (x + P - 1) // P
            lens[b], table[b, :k] = x, order[at:at + k]
            at += k
        refs = np.zeros(pages, np.int32)
        refs[order[:at]] = 1
        kids = np.arange(B, n)
        s["src"], s["dst"] = i32((kids - B) // c["branches"]), i32(kids)
        s["drop"] = i32(np.where(np.arange(n) < B, 1 << 30, 0))
        s["more"] = i32(np.where(np.arange(n) < B, 0, c["new"]))
        s["table"], s["refs"], s["lens"] = i32(table), i32(refs), i32(lens)
        _history(s, c, g, pages, P, dev)
    else:
        used = (c["fill"] + 1) // 2
        at = np.sort(rng.permutation(c["fill"])[:used])
        cols = (used + B - 1) // B
        table = np.full((B, cols), -1, np.int32)
        table.reshape(-1)[:used] = rng.permutation(at)
        refs = np.zeros(c["fill"], np.int32)
        refs[at] = rng.integers(1, 4, used)
        s["table"], s["refs"] = i32(table), i32(refs)
        s["lens"] = i32((table >= 0).sum(1) * P)
        _history(s, c, g, c["fill"], P, dev)
        s["to"] = {k: torch.zeros(used, *s[k].shape[1:], dtype=torch.uint8, device=dev) for k in PLANES}
        s["to"].update(table=torch.empty_like(s["table"]), refs=torch.empty(used, dtype=torch.int32, device=dev),
                       lens=torch.empty_like(s["lens"]))
    if own:
        from paper_2403_20137_b200 import binding as lib
        s["cache"] = lib.Cache.of(s["k_mant"], s["k_exp"], s["v_mant"], s["v_exp"], c["block"], c["bits"])
        if P:
            s["pool"] = lib.PagePool.of(s["table"], s.get("refs"), s["lens"], s["k_mant"].shape[0], P)
        if c["op"] == "attend":
            s["workspace"] = torch.empty(lib.ragged_workspace_bytes(s["cache"].fmt, B, H * G, c["new"]), dtype=torch.uint8,
                                         device=dev)
        if c["op"] == "pack":
            t = s["to"]
            s["to_cache"] = lib.Cache.of(t["k_mant"], t["k_exp"], t["v_mant"], t["v_exp"], c["block"], c["bits"])
            s["to_pool"] = lib.PagePool.of(t["table"], t["refs"], t["lens"], used, P)
    return s


# ---------------------------------------------------------------------------------------------------- the plain forms
def _values(mant, exp8, bits, block):
    """Packed rows -> fp32 values."""
    if bits == 8:
        f = mant
    elif bits == 4:
        f = torch.stack((mant & 15, mant >> 4), -1).flatten(-2)
    else:
        a, b, d = (mant[..., i::3].int() for i in range(3))
        f = torch.stack((a & 63, (a >> 6) | ((b & 15) << 2), (b >> 4) | ((d & 3) << 4), d >> 2), -1).flatten(-2)
    unit = _unit_of(exp8, bits).float()
    return ((f.float() - float(1 << (bits - 1))).reshape(*f.shape[:-1], D // block, block) * unit[..., None]).reshape(f.shape)


def _tokens(s):
    """Of every new token: its sequence, its index among the sequence's new tokens, its position."""
    starts = s["starts"].long()
    t = torch.arange(s["q_out" if "q_out" in s else "q"].shape[0], device="cuda")
    b = torch.searchsorted(starts, t, right=True) - 1
    i = t - starts[b]
    return b, i, s["lens"].long()[b] - (starts[b + 1] - starts[b]) + i


def _rotate(x, pos, theta, half, dt):
    """Rows [T, heads, D] of type dt turned by the angles of their positions (formed in 64 bits)."""
    angle = pos[:, None].double() * theta
    cs, sn = torch.cos(angle).to(dt)[:, None], torch.sin(angle).to(dt)[:, None]
    a, b = (x[..., :D // 2], x[..., D // 2:]) if half else (x[..., 0::2], x[..., 1::2])
    y = (a * cs - b * sn, a * sn + b * cs)
    return torch.cat(y, -1) if half else torch.stack(y, -1).flatten(-2)


def _write(s):
    c = s["case"]
    H, G, P = c["kv_heads"], c["group"], c["page"]
    b, _, pos = _tokens(s)
    x = s["qkv"]
    norm = lambda y, w: y * (y.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * w
    q = norm(x[:, :H * G].float(), s["q_weight"])
    s["q_out"].copy_(_rotate(q, pos, s["theta"], c["half"], torch.float32))
    # keys in 64 bits: the cast rounds to few bits, and a value next to a border has to fall on its side of it
    k = norm(x[:, H * G:H * (G + 1)].double(), s["k_weight"].double())
    k = _rotate(k, pos, s["theta"], c["half"], torch.float64)
    k = k.gather(-1, s["perm"].long().expand_as(k))
    v = x[:, H * (G + 1):].float()
    first = s["table"].long()[b, pos // P] if P else b
    row = pos % P if P else pos
    for name, y in (("k", k), ("v", v)):
        m, e = _cast(y, c["bits"], c["block"])
        s[name + "_mant"][first, :, row] = m
        s[name + "_exp"][first, :, row] = e
    return {"q": s["q_out"], **{n: _values(s[n + "_mant"], s[n + "_exp"], c["bits"], c["block"]).transpose(1, 2).bfloat16()
                                for n in ("k", "v")}}


def _rows(s, which):
    """Every sequence's rows in order, [B, H, S, D] fp32."""
    c = s["case"]
    x = _values(s[which + "_mant"], s[which + "_exp"], c["bits"], c["block"])
    if not c["page"]:
        return x
    x = x[s["table"].long().clamp_min(0)]                                        # [B, columns, H, P, D]
    return x.transpose(1, 2).flatten(2, 3)


def _attend(s):
    c = s["case"]
    B, H, G, N = c["batch"], c["kv_heads"], c["group"], c["new"]
    b, i, pos = _tokens(s)
    q = torch.zeros(B, N, H, G, D, device="cuda")
    q[b, i] = s["q"].float().reshape(-1, H, G, D).gather(-1, s["perm"].long()[None, :, None].expand(b.shape[0], H, G, D))
    at = torch.full((B, N), -1, device="cuda")
    at[b, i] = pos
    k = _rows(s, "k")
    x = q.permute(0, 2, 1, 3, 4).reshape(B, H, N * G, D) @ k.transpose(-1, -2)
    del k
    x *= 1.0 / math.sqrt(D)
    t = torch.arange(x.shape[-1], device="cuda")
    dist = at[:, :, None] - t
    seen = dist >= 0
    if c["window"]:
        seen &= (dist < c["window"]) | (t < c["sink"])
    x = x.reshape(B, H, N, G, -1).masked_fill_(~seen[:, None, :, None], float("-inf"))
    x -= x.amax(-1, keepdim=True).clamp_min(-3e38)
    p = x.exp_()
    total = p.sum(-1, keepdim=True)
    p /= torch.where(total > 0, total, 1.0)
    o = p.reshape(B, H, N * G, -1) @ _rows(s, "v")
    return o.reshape(B, H, N, G, D).permute(0, 2, 1, 3, 4).reshape(B, N, H * G, D)[b, i].to(s["q"].dtype)


def _branch(s):
    c = s["case"]
    P = c["page"]
    table, refs, lens = s["table"], s["refs"], s["lens"]
    n, cols = table.shape
    col = torch.arange(cols, device="cuda")
    held = lambda x: (x.long() + P - 1) // P
    # the branches of the step before give their pages back
    gone = (table >= 0) & (col >= held(s["drop"].clamp_max(cols * P))[:, None])
    refs.scatter_add_(0, table.clamp_min(0).long().flatten(), -gone.flatten().to(torch.int32))
    table.masked_fill_(gone, -1)
    lens.copy_(torch.minimum(lens, s["drop"]))
    # new ones share their parent's
    src, dst = s["src"].long(), s["dst"].long()
    rows = torch.where(col < held(lens[src])[:, None], table[src], -1)
    table[dst] = rows
    lens[dst] = lens[src]
    refs.scatter_add_(0, rows.clamp_min(0).long().flatten(), (rows >= 0).flatten().to(torch.int32))
    # room for what they write next: shared pages it goes to are replaced, the lowest free numbers first
    want = lens + s["more"]
    last = table.gather(1, (lens.long() // P).clamp_max(cols - 1)[:, None])[:, 0].long()
    into = (want > lens) & (lens % P > 0)
    owners = refs[last.clamp_min(0)]
    idx = torch.arange(n, device="cuda")
    same = into[None] & (last[None] == last[:, None]) & (idx[None] < idx[:, None])
    own_copy = into & (owners > 1) & (same.sum(1) != owners - 1)
    take = (col >= held(lens)[:, None]) & (col < held(want)[:, None])
    take |= own_copy[:, None] & (col == (lens.long() // P)[:, None])
    free = torch.sort((refs != 0).to(torch.int32), stable=True).indices
    rank = (take.flatten().cumsum(0) - 1).clamp_min(0)
    page = free[rank.clamp_max(free.shape[0] - 1)].reshape(n, cols).to(torch.int32)
    fits = take.sum(1).cumsum(0) <= (refs == 0).sum()
    take &= fits[:, None]
    own_copy &= fits
    refs.scatter_add_(0, page.flatten().long(), take.flatten().to(torch.int32))
    refs.scatter_add_(0, last.clamp_min(0), -own_copy.to(torch.int32))
    pairs = torch.full((n, 2), -1, dtype=torch.int32, device="cuda")
    table.copy_(torch.where(take, page, table))
    now = table.gather(1, (lens.long() // P).clamp_max(cols - 1)[:, None])[:, 0]
    pairs[:, 0] = torch.where(own_copy, last.to(torch.int32), -1)
    pairs[:, 1] = torch.where(own_copy, now, -1)
    lens.copy_(torch.where(fits, want, lens))
    some = own_copy.nonzero()[:, 0]
    a, b = pairs[some, 0].long(), pairs[some, 1].long()
    s["k_mant"][b], s["k_exp"][b] = s["k_mant"][a], s["k_exp"][a]
    s["v_mant"][b], s["v_exp"][b] = s["v_mant"][a], s["v_exp"][a]
    return pairs


def _pack(s):
    t = s["to"]
    used = s["refs"] > 0
    to = used.to(torch.int32).cumsum(0, dtype=torch.int32) - 1
    t["table"].copy_(torch.where(s["table"] >= 0, to[s["table"].clamp_min(0).long()], -1))
    at = used.nonzero()[:, 0]
    n = at.shape[0]
    t["refs"][:n] = s["refs"][at]
    t["refs"][n:] = 0
    t["lens"].copy_(s["lens"])
    t["k_mant"][:n], t["k_exp"][:n] = s["k_mant"][at], s["k_exp"][at]
    t["v_mant"][:n], t["v_exp"][:n] = s["v_mant"][at], s["v_exp"][at]


def run(state):
    s = state
    c = s["case"]
    if own:
        from paper_2403_20137_b200 import binding as lib
    if c["op"] == "write":
        if not own:
            return _write(s)
        x, hq, hk = s["qkv"], c["kv_heads"] * c["group"], c["kv_heads"]
        lib.norm_rope_append(s["cache"], x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:], s["starts"], s["lens"],
                             q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6, theta=s["theta"], half_split=c["half"],
                             perm_k=s["perm"], pool=s.get("pool"), q_out=s["q_out"])
        rows = s["k_mant"].shape[2]
        return {"q": s["q_out"], **{n: lib.dequant_all(s["cache"], n, rows, out_dtype=torch.bfloat16) for n in ("k", "v")}}
    if c["op"] == "attend":
        if not own:
            return _attend(s)
        return lib.ragged_attn(s["cache"], s["q"], s["starts"], s["lens"], c["new"], window=c["window"], n_sink=c["sink"],
                               perm_k=s["perm"], pool=s.get("pool"), workspace=s["workspace"])
    if c["op"] == "branch":
        if own:
            lib.pages_free(s["pool"], lo=s["drop"])
            lib.pages_fork(s["pool"], s["src"], s["dst"])
            pairs = lib.pages_reserve(s["pool"], s["more"])
            lib.pages_copy(s["cache"], pairs)
        else:
            pairs = _branch(s)
        return {"pairs": pairs, **{k: s[k] for k in ("table", "refs", "lens") + PLANES}}
    if own:
        moves, count = lib.pages_compact(s["pool"], dst=s["to_pool"])
        lib.pages_copy(s["cache"], moves, count=count, dst=s["to_cache"])
    else:
        _pack(s)
    return s["to"]


# ---------------------------------------------------------------------------------------------------- in 64 bits
def _exact_values(mant, exp8, bits, block):
    """Packed rows [n, bytes] -> fp64 [n, D], field by field from the bit stream."""
    raw = torch.nn.functional.pad(mant.to(torch.int64), (0, 1))
    bit = torch.arange(D, device=mant.device) * bits
    f = ((raw[:, bit // 8] | (raw[:, bit // 8 + 1] << 8)) >> (bit % 8)) & ((1 << bits) - 1)
    e = exp8.double()[:, torch.arange(D, device=mant.device) // block] - 127.0 - (bits - 2)
    return (f.double() - 2.0 ** (bits - 1)) * torch.pow(torch.tensor(2.0, dtype=torch.float64, device=mant.device), e)


def _exact_attend(s, c):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for b, (n, new) in enumerate(zip(_lens(c), _news(c))):
        at = torch.arange(n, device="cuda")
        pos = torch.arange(n - new, n, device="cuda")[:, None]
        see = at <= pos
        if c["window"]:
            see &= (at > pos - c["window"]) | (at < c["sink"])
        for h in range(c["kv_heads"]):
            if c["page"]:
                pages = s["table"][b].long()[at // c["page"]]
                k, v = (_exact_values(s[w + "_mant"][pages, h, at % c["page"]], s[w + "_exp"][pages, h, at % c["page"]],
                                      c["bits"], c["block"]) for w in ("k", "v"))
            else:
                k, v = (_exact_values(s[w + "_mant"][b, h, :n], s[w + "_exp"][b, h, :n], c["bits"], c["block"])
                        for w in ("k", "v"))
            channels = torch.empty_like(k)
            channels[:, s["perm"][h].long()] = k
            for hq in range(h * c["group"], (h + 1) * c["group"]):
                x = s["q"][row:row + new, hq].double() @ channels.T / D ** 0.5
                out[row:row + new, hq] = torch.softmax(torch.where(see, x, -math.inf), -1) @ v
        row += new
    return out


def _exact_write(s, c):
    """Token by token of a sequence: complex rotation, and the cast as the nearest multiple of the block's unit."""
    H, G, P, half = c["kv_heads"], c["group"], c["page"], c["half"]
    x = s["qkv"].double()
    pos = torch.cat([torch.arange(n - m, n, device="cuda") for n, m in zip(_lens(c), _news(c))]).double()
    seq = torch.cat([torch.full((m,), b, device="cuda") for b, m in enumerate(_news(c))])
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.outer(pos, s["theta"]))[:, None]

    def rotated(y, w):
        y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / D + 1e-6) * w.double()
        z = (torch.complex(y[..., :D // 2], y[..., D // 2:]) if half else torch.view_as_complex(y.reshape(*y.shape[:-1], D // 2, 2).contiguous())) * turn
        return torch.cat((z.real, z.imag), -1) if half else torch.view_as_real(z).reshape(y.shape)

    out = {"q": rotated(x[:, :H * G], s["q_weight"])}
    for name, y in (("k", rotated(x[:, H * G:H * (G + 1)], s["k_weight"])), ("v", x[:, H * (G + 1):])):
        if name == "k":
            y = torch.stack([y[:, h, s["perm"][h].long()] for h in range(H)], 1)
        blocks = y.reshape(*y.shape[:-1], D // c["block"], c["block"])
        most = blocks.abs().amax(-1, keepdim=True)
        unit = 2.0 ** torch.floor(torch.log2(most * (1 + 2.0 ** -50))) / 2.0 ** (c["bits"] - 2)
        top = 2.0 ** (c["bits"] - 1) - 1
        y = (torch.round(blocks / unit).clamp(-top, top) * unit).reshape(y.shape)
        shape = s[name + "_mant"].shape
        old = torch.cat([_exact_values(m.reshape(-1, m.shape[-1]), e.reshape(-1, e.shape[-1]), c["bits"], c["block"])
                         for m, e in zip(s[name + "_mant"].split(64), s[name + "_exp"].split(64))]).reshape(*shape[:3], D).transpose(1, 2)
        where = s["table"].long()[seq, (pos // P).long()] if P else seq
        old[where, (pos % P).long() if P else pos.long()] = y
        out[name] = old
    return out


def exact(case, seed):
    c = case
    if c["op"] == "attend":
        return _exact_attend(prepare(case, seed), c)
    if c["op"] == "write":
        return _exact_write(prepare(case, seed), c)
    return None
