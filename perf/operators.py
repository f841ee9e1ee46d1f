"""Cases of the cache operators beyond plain decoding: attention of a tree of drafted tokens over the packed cache,
decode attention with capped scores, distance bias and masks, decode attention that accumulates each token's attention
weight, eviction by that weight, and the row move that commits an accepted branch.

The packed cache (block floating point) is made here from seeded values: blocks of ``block`` slots share an exponent
byte E + 127, a slot holds M + 2^(bits-1) in ``bits`` bits of a little-endian stream, its value is M 2^(E-(bits-2)).
"""
import math

import numpy as np
import torch

own = False

D = 128


# ---------------------------------------------------------------------------------------------------- the cases
def _case(name, op, batch, kv_heads, group, seq, bits, block, dtype, **more):
    c = {"name": name, "op": op, "batch": batch, "kv_heads": kv_heads, "group": group, "seq": seq, "bits": bits,
         "block": block, "dtype": dtype, "ragged": False, "draft": 0, "chain": False, "cap": 0.0, "bias": False,
         "window": 0, "prefix": 0, "doc": False, "budget": 0, "sink": 0, "recent": 0}
    c.update(more)
    return c


def listed():
    return [
        # one fp32 head over a short cache, a handful of drafted tokens: the smallest call, all latency
        _case("tree tiny f32", "tree", 1, 1, 1, 256, 4, 16, "f32", draft=5),
        # one user, 32 heads, a chain of 8 drafted tokens checked at once
        _case("tree b1 h32 chain 8", "tree", 1, 32, 1, 4096, 4, 32, "bf16", draft=8, chain=True),
        # a batch of users with ragged histories, a tree of 16 each
        _case("tree b16 h32 t16", "tree", 16, 32, 1, 8192, 4, 32, "bf16", draft=16, ragged=True),
        # grouped heads over long histories, a tree of 16: 64 query rows read every cached row
        _case("tree b8 gqa t16", "tree", 8, 8, 4, 32768, 4, 32, "bf16", draft=16),
        # grouped heads, 8-bit cache, the widest tree: 256 query rows
        _case("tree b8 gqa t64 8bit", "tree", 8, 8, 4, 8191, 8, 32, "bf16", draft=64, cap=50.0, ragged=True),
        # one user, capped scores and a sliding window with its first tokens kept visible
        _case("mod b1 h32 window", "mod", 1, 32, 1, 4096, 4, 32, "bf16", cap=30.0, window=1000, prefix=4),
        # grouped heads, distance bias, histories that begin with another document
        _case("mod b8 gqa bias doc", "mod", 8, 8, 4, 32768, 4, 32, "bf16", bias=True, doc=True, ragged=True),
        # weights gathered over a ragged fp32 batch with 6-bit rows
        _case("mass b2 gqa f32 6bit", "mass", 2, 2, 4, 1003, 6, 16, "f32", ragged=True, cap=20.0),
        # weights gathered in a batch of users
        _case("mass b16 h32", "mass", 16, 32, 1, 8192, 4, 32, "bf16"),
        # a long prompt cut down to what it attended to
        _case("evict b1 h8 64k", "evict", 1, 8, 1, 65536, 4, 32, "bf16", budget=4096, sink=16, recent=512),
        # a batch of users cut back, some of them short enough to stay whole
        _case("evict b16 h32 8k", "evict", 16, 32, 1, 8192, 4, 32, "bf16", budget=2048, sink=4, recent=256, ragged=True),
        # the accepted branches of a batch's trees moved together
        _case("commit b16 h32 t64", "commit", 16, 32, 1, 1024, 4, 32, "bf16", draft=64),
        ]


def draw(rng):
    """Any operator, sizes from one token to the largest listed work, every format."""
    op = rng.choice(["tree", "tree", "tree", "mod", "mod", "mass", "evict", "commit"])
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    batch = log(1, 16)
    kv_heads = rng.choice([1, 2, 3, 4, 8, 8, 16, 32])
    group = rng.choice([1, 1, 2, 3, 4, 4, 5, 8]) if op in ("tree", "mod", "mass") else 1
    top = {"tree": 1 << 21, "mod": 1 << 21, "mass": 1 << 21, "evict": 1 << 21, "commit": 1 << 19}[op]
    draft = log(1, 64) if op in ("tree", "commit") else 0
    if op == "tree":                        # rows times units: no more than the largest listed
        top = min(top, (1 << 27) // max(1, draft * group))
    seq = log(1, max(1, min(65536 if op == "evict" else 32768, top // (batch * kv_heads))))
    c = _case("", op, batch, kv_heads, group, seq, rng.choice([4, 4, 4, 6, 8]), rng.choice([16, 32, 32, 64, 128]),
              rng.choice(["bf16", "bf16", "f32"]), ragged=rng.random() < 0.5, draft=draft)
    del c["name"]
    if op == "tree":
        c["chain"] = rng.random() < 0.3
    if op in ("tree", "mod", "mass"):
        c["cap"] = rng.choice([0.0, 0.0, 20.0, 50.0])
        c["bias"] = rng.random() < 0.3
        if rng.random() < 0.4:
            c["window"] = log(1, max(1, seq))
            c["prefix"] = rng.choice([0, 4, 100])
        c["doc"] = rng.random() < 0.3
    if op == "evict":
        c["budget"] = max(1, log(1, seq))
        c["sink"] = rng.randint(0, min(16, c["budget"]))
        c["recent"] = rng.randint(0, (c["budget"] - c["sink"]) // 2)
    return c


def _lens(c):
    """Cached tokens of each sequence (for a tree: before the drafted ones); the first is the longest."""
    if c["op"] == "commit":
        return [max(0, c["seq"] - (7 * b) % 64) for b in range(c["batch"])]
    if not c["ragged"]:
        return [c["seq"]] * c["batch"]
    return [c["seq"] - (c["seq"] * ((b * 37) % 64)) // 80 for b in range(c["batch"])]


def _drafts(c):
    """Drafted tokens of each sequence."""
    if not c["ragged"]:
        return [c["draft"]] * c["batch"]
    return [max(1, c["draft"] - (b * 5) % (c["draft"] // 2 + 1)) for b in range(c["batch"])]


def _firsts(c):
    return [n // 4 for n in _lens(c)]


def _paths(c):
    """Accepted branch lengths of each sequence."""
    return [1 + (b * 11 + c["draft"] // 2) % c["draft"] for b in range(c["batch"])]


def _seen(c):
    """Cached tokens (of one head) that any query of a sequence sees, summed over the batch."""
    total = 0
    for n, first in zip(_lens(c), _firsts(c)):
        lo = first if c["doc"] else 0
        if c["window"]:
            lo = max(lo, n - c["window"] + (0 if c["op"] != "tree" else 1))
        lo = min(max(lo, 0), n)
        total += n - lo + min(c["prefix"] if (c["window"] or c["doc"]) else 0, lo)
    return total


def _unit(c):
    return 2 * (D * c["bits"] // 8 + D // c["block"])


def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    heads = c["kv_heads"] * c["group"]
    if c["op"] in ("tree", "mod", "mass"):
        t = c["draft"] if c["op"] == "tree" else 1
        seen = _seen(c) + (sum(_drafts(c)) if c["op"] == "tree" else 0)
        by = seen * c["kv_heads"] * _unit(c) + 2 * c["batch"] * t * heads * D * es
        rows = seen * heads * (sum(_drafts(c)) / c["batch"] if c["op"] == "tree" else 1)
        if c["op"] == "mass":
            by += 8 * seen * c["kv_heads"]
        return {"bytes": by, "flops": 4 * D * rows}
    if c["op"] == "evict":
        kept = sum(min(n, c["budget"]) for n in _lens(c)) * c["kv_heads"]
        return {"bytes": 4 * sum(_lens(c)) * c["kv_heads"] + kept * (2 * _unit(c) + 8), "flops": 0}
    return {"bytes": 2 * sum(_paths(c)) * c["kv_heads"] * _unit(c), "flops": 0}


# ---------------------------------------------------------------------------------------------------- the inputs
def _weights(bits, device, dtype=torch.float32):
    """Value of one mantissa unit for each exponent byte."""
    return torch.tensor([2.0 ** (e - 127 - (bits - 2)) for e in range(256)], dtype=torch.float64).to(device=device, dtype=dtype)


def _pack(x, bits, block):
    """Values [..., D] -> mantissa bytes [..., D * bits / 8], exponent bytes [..., D / block]."""
    blocks = x.float().reshape(*x.shape[:-1], D // block, block)
    e8 = (blocks.abs().amax(-1).view(torch.int32) >> 23) & 255
    unit = _weights(bits, x.device)[e8.long()]
    top = (1 << (bits - 1)) - 1
    f = (torch.round(blocks / unit[..., None]).clamp(-top, top).to(torch.int32) + (1 << (bits - 1))).reshape(x.shape)
    if bits == 8:
        m = f
    elif bits == 4:
        m = f[..., 0::2] | (f[..., 1::2] << 4)
    else:
        w = f[..., 0::4] | (f[..., 1::4] << 6) | (f[..., 2::4] << 12) | (f[..., 3::4] << 18)
        m = torch.stack((w & 255, (w >> 8) & 255, w >> 16), -1).flatten(-2)
    return m.to(torch.uint8).contiguous(), e8.to(torch.uint8).contiguous()


def _tree(c, rng):
    """Ancestor masks [B, T] (bit j of row i: token i sees token j) and depths [B, T] of seeded trees."""
    masks, depths = [], []
    for n in _drafts(c):
        m, d = [], []
        for i in range(c["draft"]):
            if i == 0 or i >= n:
                m.append(1 << i)
                d.append(0)
                continue
            up = i - 1 if c["chain"] else int(rng.integers(max(0, i - 8), i))
            m.append(m[up] | (1 << i))
            d.append(d[up] + 1)
        masks.append(m)
        depths.append(d)
    to = lambda v: torch.from_numpy(np.array(v, dtype=np.uint64).astype(np.int64))
    return to(masks), torch.tensor(depths, dtype=torch.int32)


def prepare(case, seed):
    c = case
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    B, H, G = c["batch"], c["kv_heads"], c["group"]
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    max_seq = (c["seq"] + c["draft"] + 15) // 16 * 16
    # a few loud key channels per head, found by the calibration as an order of the channels
    scale = torch.ones(H, D)
    for h in range(H):
        scale[h, torch.from_numpy(rng.permutation(D)[:6])] = torch.from_numpy(np.exp(rng.normal(1.5, 0.4, 6))).float()
    scale = scale.to(dev)
    perm = torch.sort(scale + 0.01 * torch.rand(H, D, generator=g, device=dev), dim=-1, stable=True).indices
    planes = {"k": ([], []), "v": ([], [])}
    for _ in range(B):
        for which in ("k", "v"):
            x = torch.randn(H, max_seq, D, generator=g, device=dev)
            if which == "k":
                x = (x * scale[:, None]).gather(-1, perm[:, None].expand_as(x))
            for to, p in zip(planes[which], _pack(x, c["bits"], c["block"])):
                to.append(p)
    s = {"case": c, "max_seq": max_seq, "perm": perm.to(torch.int32).contiguous(),
         "k_mant": torch.stack(planes["k"][0]), "k_exp": torch.stack(planes["k"][1]),
         "v_mant": torch.stack(planes["v"][0]), "v_exp": torch.stack(planes["v"][1]),
         "lens": torch.tensor(_lens(c), dtype=torch.int32, device=dev)}
    if c["op"] in ("tree", "mod", "mass"):
        shape = (B, c["draft"], H * G, D) if c["op"] == "tree" else (B, H * G, D)
        s["q"] = torch.randn(shape, generator=g, device=dev).to(dt)
        s["first"] = torch.tensor(_firsts(c), dtype=torch.int32, device=dev) if c["doc"] else None
        s["prefix"] = torch.full((B,), c["prefix"], dtype=torch.int32, device=dev) if c["prefix"] else None
        s["slopes"] = (2.0 ** (-8.0 * torch.arange(1, H * G + 1, device=dev) / (H * G))).float() if c["bias"] else None
    if c["op"] == "tree":
        mask, depth = _tree(c, rng)
        s["mask"], s["depth"] = mask.to(dev), depth.to(dev)
        s["drafts"] = torch.tensor(_drafts(c), dtype=torch.int32, device=dev)
    if c["op"] in ("mass", "evict"):
        # weights as softmax leaves them: a few tokens hold most, none where no token is
        m = torch.exp(2.0 * torch.randn(B, H, max_seq, generator=g, device=dev) - 4.0)
        if c["op"] == "evict":
            m = torch.round(m * 4096.0) / 4096.0            # equal weights too: the lower position is kept
        s["mass"] = torch.where(torch.arange(max_seq, device=dev) < s["lens"][:, None, None], m, 0.0).contiguous()
    if c["op"] == "evict":
        rows = (c["budget"] + 15) // 16 * 16
        s["to"] = {k: torch.zeros(B, H, rows, s[k].shape[-1], dtype=torch.uint8, device=dev)
                   for k in ("k_mant", "k_exp", "v_mant", "v_exp")}
        s["to_mass"] = torch.zeros(B, H, rows, device=dev)
    if c["op"] == "commit":
        idx = np.zeros((B, c["draft"]), np.int32)
        for b, n in enumerate(_paths(c)):
            idx[b, :n] = np.sort(rng.permutation(c["draft"])[:n])
        s["index"] = torch.from_numpy(idx).to(dev)
        s["count"] = torch.tensor(_paths(c), dtype=torch.int32, device=dev)
    if own:
        from paper_2403_20137_b200 import binding as lib
        s["cache"] = _cache(lib, s, c, max_seq, s)
        if c["op"] == "evict":
            s["to_cache"] = _cache(lib, s["to"], c, s["to"]["k_mant"].shape[2], s)
        if c["op"] in ("tree", "mod", "mass"):
            s["mod"] = lib.ScoreMod(softcap=c["cap"], slopes=s["slopes"], first=s["first"], prefix=s["prefix"],
                                    window=c["window"])
            s["workspace"] = torch.empty(lib.attn_workspace_bytes(s["cache"].fmt, H * G, max(1, c["draft"]),
                                                                  c["op"] == "mass"), dtype=torch.uint8, device=dev)
    return s


def _cache(lib, planes, c, max_seq, s):
    cache = lib.Cache.__new__(lib.Cache)
    cache.fmt = lib.Format(c["batch"], c["kv_heads"], D, max_seq, c["block"], c["bits"])
    for k in ("k_mant", "k_exp", "v_mant", "v_exp"):
        setattr(cache, k, planes[k])
    return cache


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
    unit = _weights(bits, mant.device)[exp8.long()]
    return ((f.float() - float(1 << (bits - 1))).reshape(*f.shape[:-1], D // block, block) * unit[..., None]).reshape(f.shape)


def _visible(s, T):
    """(visible [B, T, S], distance [B, T, S]) of every query and cached row."""
    c = s["case"]
    S = s["max_seq"]
    t = torch.arange(S, device="cuda")
    n = s["lens"].long()[:, None, None]
    if c["op"] == "tree":
        depth = s["depth"].long()
        pos_q = n + depth[:, :, None]
        j = (t - n).clamp(0, T - 1)                                              # [B, 1, S]
        drafted = (t >= n) & (t < n + s["drafts"].long()[:, None, None])
        pos_k = torch.where(drafted, n + depth.gather(1, j[:, 0]).unsqueeze(1), t)
        seen_draft = drafted & (((s["mask"][:, :, None] >> j) & 1) == 1)
    else:
        pos_q = (n - 1).expand(-1, 1, 1)
        pos_k = t.expand(n.shape[0], 1, S)
        drafted = seen_draft = torch.zeros_like(pos_k, dtype=torch.bool)
    dist = pos_q - pos_k
    near = dist < c["window"] if c["window"] else torch.ones_like(dist, dtype=torch.bool)
    ctx = near if s["first"] is None else near & (t >= s["first"].long()[:, None, None])
    if s["prefix"] is not None:
        ctx = ctx | (t < s["prefix"].long()[:, None, None])
    seen = torch.where(drafted, seen_draft & near, ctx & (t < n))
    if c["op"] == "tree":
        seen = seen & (torch.arange(T, device="cuda")[None, :, None] < s["drafts"].long()[:, None, None])
    return seen, dist


def _attention(s):
    """(out [B, T, Hq, D] of q's type, weights [B, Hkv, T * G, S] fp32)."""
    c = s["case"]
    B, H, G = c["batch"], c["kv_heads"], c["group"]
    q = s["q"] if c["op"] == "tree" else s["q"][:, None]
    T = q.shape[1]
    k = _values(s["k_mant"], s["k_exp"], c["bits"], c["block"])
    qf = q.float().reshape(B, T, H, G, D).gather(-1, s["perm"].long()[None, None, :, None].expand(B, T, H, G, D))
    qf = qf.permute(0, 2, 1, 3, 4).reshape(B, H, T * G, D)
    x = (qf @ k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    del k
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    seen, dist = _visible(s, T)
    x = x.reshape(B, H, T, G, -1)
    if s["slopes"] is not None:
        x = x - s["slopes"].reshape(1, H, 1, G, 1) * dist[:, None, :, None].float()
    x = x.masked_fill(~seen[:, None, :, None], float("-inf"))
    p = torch.exp(x - x.amax(-1, keepdim=True).clamp_min(-3e38))
    total = p.sum(-1, keepdim=True)
    p = (p / torch.where(total > 0, total, 1.0)).reshape(B, H, T * G, -1)
    o = p @ _values(s["v_mant"], s["v_exp"], c["bits"], c["block"])
    o = o.reshape(B, H, T, G, D).permute(0, 2, 1, 3, 4).reshape(B, T, H * G, D)
    return o.to(s["q"].dtype), p


def _evict(s):
    c = s["case"]
    S, K = s["max_seq"], c["budget"]
    t = torch.arange(S, device="cuda")
    n = s["lens"].long()[:, None, None]
    mass = s["mass"].masked_fill(t >= n, float("-inf"))
    mass = mass.masked_fill(((t < c["sink"]) | (t >= n - c["recent"])) & (t < n), float("inf"))
    order = torch.sort(mass, dim=-1, descending=True, stable=True).indices[..., :K]
    kept = torch.sort(order, dim=-1).values
    slot = torch.arange(K, device="cuda")
    new = n.clamp_max(K)
    kept = torch.where(n <= K, slot[:kept.shape[-1]].clamp_max(S - 1), kept)
    kept = torch.nn.functional.pad(kept, (0, K - kept.shape[-1]))
    valid = slot < new                                                           # [B, 1, K]
    for k, dst in s["to"].items():
        rows = s[k].gather(2, kept[..., None].expand(*kept.shape, s[k].shape[-1]))
        dst[:, :, :K] = torch.where(valid[..., None], rows, dst[:, :, :K])
    s["to_mass"][:, :, :K] = torch.where(valid, s["mass"].gather(2, kept), 0.0)
    s["to_mass"][:, :, K:] = 0.0
    return torch.where(valid, kept, -1).to(torch.int32), new[:, 0, 0].to(torch.int32)


def _commit(s):
    c = s["case"]
    T = c["draft"]
    i = torch.arange(T, device="cuda")
    at = s["lens"].long()[:, None] + i                                           # [B, T]
    src = torch.where(i < s["count"].long()[:, None], s["lens"].long()[:, None] + s["index"].long(), at)
    for k in ("k_mant", "k_exp", "v_mant", "v_exp"):
        p = s[k]
        grow = lambda x: x[:, None, :, None].expand(p.shape[0], p.shape[1], T, p.shape[3])
        p.scatter_(2, grow(at), p.gather(2, grow(src)))


def run(state):
    s = state
    c = s["case"]
    if own:
        from paper_2403_20137_b200 import binding as lib
    if c["op"] == "tree":
        if own:
            return lib.tree_attn(s["cache"], s["q"], s["lens"], draft_lens=s["drafts"], tree_mask=s["mask"], depth=s["depth"],
                                 perm_k=s["perm"], mod=s["mod"], workspace=s["workspace"])
        return _attention(s)[0]
    if c["op"] == "mod":
        if own:
            return lib.decode_attn_mod(s["cache"], s["q"], s["lens"], s["mod"], perm_k=s["perm"], workspace=s["workspace"])
        return _attention(s)[0][:, 0]
    if c["op"] == "mass":
        if own:
            out = lib.decode_attn_mass(s["cache"], s["q"], s["lens"], s["mass"], mod=s["mod"], perm_k=s["perm"],
                                       workspace=s["workspace"])
        else:
            out, p = _attention(s)
            out = out[:, 0]
            s["mass"] += p.sum(2)
        return {"out": out, "mass": s["mass"]}
    if c["op"] == "evict":
        if own:
            kept, new = lib.evict(s["cache"], s["lens"], s["mass"], c["budget"], c["sink"], c["recent"], dst=s["to_cache"],
                                  dst_mass=s["to_mass"])
        else:
            kept, new = _evict(s)
        return {"kept": kept, "lens": new, "mass": s["to_mass"], **s["to"]}
    if own:
        lib.gather_rows(s["cache"], s["index"], s["count"], s["lens"])
    else:
        _commit(s)
    lo = max(0, c["seq"] - 64)
    return {k: s[k][:, :, lo:] for k in ("k_mant", "k_exp", "v_mant", "v_exp")}


# ---------------------------------------------------------------------------------------------------- in 64 bits
def _exact_values(mant, exp8, bits, block):
    """One head's packed rows [n, bytes] -> fp64 [n, D], field by field from the bit stream."""
    raw = torch.nn.functional.pad(mant.to(torch.int64), (0, 1))
    bit = torch.arange(D, device=mant.device) * bits
    f = ((raw[:, bit // 8] | (raw[:, bit // 8 + 1] << 8)) >> (bit % 8)) & ((1 << bits) - 1)
    e = exp8.double()[:, torch.arange(D, device=mant.device) // block] - 127.0 - (bits - 2)
    return (f.double() - 2.0 ** (bits - 1)) * torch.pow(torch.tensor(2.0, dtype=torch.float64, device=mant.device), e)


def _exact_attention(s, c):
    B, H, G = c["batch"], c["kv_heads"], c["group"]
    tree = c["op"] == "tree"
    q = s["q"].double() if tree else s["q"].double()[:, None]
    T = q.shape[1]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    mass = s["mass"].double().clone() if c["op"] == "mass" else None
    lens, drafts = _lens(c), _drafts(c) if tree else [1] * B
    for b in range(B):
        n, nd = lens[b], drafts[b]
        rows = n + (nd if tree else 0)
        if rows == 0:
            continue
        # positions, and who sees whom, token by token of the draft
        key = list(range(n))
        depth = s["depth"][b].tolist() if tree else [-1]
        pk = torch.tensor(key + [n + depth[j] for j in range(nd if tree else 0)], dtype=torch.float64, device="cuda")
        see = torch.zeros(nd, rows, dtype=torch.bool, device="cuda")
        dist = torch.zeros(nd, rows, dtype=torch.float64, device="cuda")
        for i in range(nd):
            dist[i] = float(n + depth[i]) - pk
            ok = torch.ones(rows, dtype=torch.bool, device="cuda")
            if c["window"]:
                ok &= dist[i] < c["window"]
            if c["doc"]:
                ok[:min(_firsts(c)[b], n)] = False
            if c["prefix"]:
                ok[:min(c["prefix"], n)] = True
            if tree:
                bits = int(s["mask"][b, i]) & ((1 << 64) - 1)
                for j in range(nd):
                    if not (bits >> j) & 1:
                        ok[n + j] = False
            see[i] = ok
        for h in range(H):
            k = _exact_values(s["k_mant"][b, h, :rows], s["k_exp"][b, h, :rows], c["bits"], c["block"])
            v = _exact_values(s["v_mant"][b, h, :rows], s["v_exp"][b, h, :rows], c["bits"], c["block"])
            for g in range(G):
                hq = h * G + g
                x = torch.einsum("id,td->it", q[b, :nd, hq][:, s["perm"][h].long()], k) / D ** 0.5
                if c["cap"]:
                    x = torch.tanh(x / c["cap"]) * c["cap"]
                if c["bias"]:
                    x = x - 2.0 ** (-8.0 * (hq + 1) / (H * G)) * dist if s["slopes"] is None else x - s["slopes"][hq].double() * dist
                x = torch.where(see, x, torch.full_like(x, -math.inf))
                w = torch.where(see.any(-1, keepdim=True), torch.softmax(x, -1), torch.zeros_like(x))
                out[b, :nd, hq] = w @ v
                if mass is not None:
                    mass[b, h, :rows] += w[0]
    if tree:
        return out
    return {"out": out[:, 0], "mass": mass} if mass is not None else out[:, 0]


def exact(case, seed):
    c = case
    if c["op"] == "commit":
        return None
    s = prepare(case, seed)
    if c["op"] == "evict":
        mass, to = s["mass"].cpu().numpy().astype(np.float64), np.zeros(s["to_mass"].shape)
        for b, n in enumerate(_lens(c)):
            for h in range(c["kv_heads"]):
                at = list(range(n))
                if n > c["budget"]:
                    mid = np.arange(c["sink"], n - c["recent"])
                    best = mid[np.argsort(-mass[b, h, mid], kind="stable")[:c["budget"] - c["sink"] - c["recent"]]]
                    at = np.concatenate([np.arange(c["sink"]), np.sort(best), np.arange(n - c["recent"], n)]).astype(int)
                to[b, h, :len(at)] = mass[b, h, at]
        return {"kept": None, "lens": None, "mass": to, "k_mant": None, "k_exp": None, "v_mant": None, "v_exp": None}
    return _exact_attention(s, c)
