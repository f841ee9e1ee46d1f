"""Tree attention, masked / capped / biased decode attention, attention weights, eviction and row moves over the packed
cache, against plain forms in 64 bits on the dequantised cache (whose bytes other tests pin)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2403_20137_b200 import binding as B

D = 128
FMT = [(4, 16), (4, 32), (4, 128), (6, 32), (6, 64), (8, 16), (8, 32)]
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step, relative


# ----------------------------------------------------------------------------------------------- helpers
def make_cache(batch, heads, max_seq, bits, block, seed, scale=1.0, fill=None):
    """A cache whose rows 0..max_seq-1 are all written (seeded values, a few loud channels)."""
    g = torch.Generator().manual_seed(seed)
    k = torch.randn(batch, max_seq, heads, D, generator=g) * scale
    v = torch.randn(batch, max_seq, heads, D, generator=g) * scale
    k[..., [3, 77, 120]] *= 4.0
    perm = torch.stack([torch.randperm(D, generator=g) for _ in range(heads)]).to(torch.int32).cuda()
    perm_v = torch.stack([torch.randperm(D, generator=g) for _ in range(heads)]).to(torch.int32).cuda()
    cache = B.Cache(batch, heads, D, max_seq, block, bits, fill=fill)
    B.append(cache, k.cuda(), v.cuda(), torch.zeros(batch, dtype=torch.int32, device="cuda"), perm_k=perm, perm_v=perm_v)
    return cache, perm, perm_v


def inverse(perm):
    inv = torch.empty_like(perm)
    inv.scatter_(1, perm.long(), torch.arange(D, dtype=torch.int32, device=perm.device).expand_as(perm))
    return inv


def trees(batch, T, drafts, seed, chain=False):
    rng = np.random.default_rng(seed)
    mask, depth = np.zeros((batch, T), np.uint64), np.zeros((batch, T), np.int32)
    for b in range(batch):
        for i in range(T):
            up = -1 if i == 0 else (i - 1 if chain else int(rng.integers(-1, i)))
            mask[b, i] = np.uint64(1 << i) | (mask[b, up] if up >= 0 else np.uint64(0))
            depth[b, i] = depth[b, up] + 1 if up >= 0 else 0
    return torch.from_numpy(mask.view(np.int64)).cuda(), torch.from_numpy(depth).cuda()


def reference(cache, q, lens, perm, perm_v, mod, scale=0.0, drafts=None, mask=None, depth=None):
    """-> out, the sum of p|v| per output, the sum of |q k| scale per row (largest), weights; all fp64.
    q [B, T, Hq, D]; drafts None: a single token at lens - 1."""
    f = cache.fmt
    Bn, T, Hq, _ = q.shape
    H, G = f.n_kv_heads, Hq // f.n_kv_heads
    k = B.dequant_all(cache, "k", f.max_seq, perm=perm).double()
    v = B.dequant_all(cache, "v", f.max_seq, perm=perm_v).double()
    out = torch.zeros(Bn, T, Hq, D, dtype=torch.float64, device="cuda")
    amp, reach = torch.zeros_like(out), torch.zeros(Bn, T, Hq, dtype=torch.float64, device="cuda")
    weights = torch.zeros(Bn, H, f.max_seq, dtype=torch.float64, device="cuda")
    scale = scale or 1.0 / math.sqrt(D)
    for b in range(Bn):
        n = min(max(int(lens[b]), 0), f.max_seq)
        nd = 0 if drafts is None else min(int(drafts[b]), f.max_seq - n)
        pk = torch.arange(f.max_seq, device="cuda")
        for i in range(T if drafts is None else nd):
            pos = n - 1 if drafts is None else n + int(depth[b, i])
            kp = pk.clone()
            if nd:
                kp[n:n + nd] = n + depth[b, :nd].long()
            see = pk < n
            near = (pos - kp < mod.window) if mod.window else torch.ones_like(see)
            see &= near
            if mod.first is not None:
                see &= pk >= min(max(int(mod.first[b]), 0), n)
            if mod.prefix is not None:
                see |= pk < min(max(int(mod.prefix[b]), 0), n)
            for j in range(nd):
                see[n + j] = bool((int(mask[b, i]) >> j) & 1) and bool(near[n + j])
            if not bool(see.any()):
                continue
            for hq in range(Hq):
                h = hq // G
                prod = q[b, i, hq].double() * k[b, :, h]
                x = prod.sum(-1) * scale
                reach[b, i, hq] = (prod.abs().sum(-1) * scale)[see].max()
                if mod.softcap:
                    x = mod.softcap * torch.tanh(x / mod.softcap)
                if mod.slopes is not None:
                    x = x - mod.slopes[hq].double() * (pos - kp)
                p = torch.softmax(x.masked_fill(~see, -math.inf), -1)
                out[b, i, hq] = p @ v[b, :, h]
                amp[b, i, hq] = p @ v[b, :, h].abs()
                weights[b, h] += p
    return out, amp, reach, weights


def check(got, out, amp, reach, cap=0.0, dt=None):
    """Error bound per output.  Scores: fp32 products in chains of up to 24 tensor-core steps that cut (2^-23 of the
    running sum of |q k| each; fp32 queries drop 2^-25 of q), the cap adds 2^-21 of itself; a score error d changes a
    weight by d relative, an output by 2 d sum(p|v|).  Weights are rounded to bf16 (half a step) or, for fp32
    queries, cut to three bf16 terms (2^-16 allows for two), exp2 and the sums add 2^-20; the output is rounded once."""
    d = 24 * 2.0 ** -23 * reach + cap * 2.0 ** -21
    w = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -16
    bound = amp * (2 * d[..., None] + w + 2.0 ** -20) * 1.01 + HALF[got.dtype] * out.abs() * 1.01 + 1e-35
    err = (got.double() - out).abs()
    worst = float((err / bound).max())
    finite = bool(torch.isfinite(got).all())
    assert finite and worst <= 1.0, f"error is {worst:.3g} of the bound"


def case(seed, batch, heads, group, max_seq, T, dtype, bits, block):
    cache, perm, perm_v = make_cache(batch, heads, max_seq, bits, block, seed)
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn(batch, T, heads * group, D, generator=g).to(dtype).cuda()
    return cache, perm, perm_v, q


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ----------------------------------------------------------------------------------------------- tree attention
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits,block", FMT)
@pytest.mark.parametrize("T,group", [(1, 1), (5, 1), (7, 3), (16, 1), (6, 4), (11, 5), (64, 1), (33, 4)])
def test_tree_attn_formats_and_sizes(bits, block, T, group, dtype):
    """Every format and row tile; ragged contexts, one empty, ragged drafts, both permutations."""
    if T * group > 40 and block != 32:
        pytest.skip("the widest trees run on one block size per width")
    cache, perm, perm_v, q = case(T * 7 + group, 3, 2, group, 448, T, dtype, bits, block)
    lens, drafts = i32(300, 0, 129), i32(T, max(1, T // 2), T)
    mask, depth = trees(3, T, drafts, 5)
    mod = B.ScoreMod()
    got = B.tree_attn(cache, q, lens, draft_lens=drafts, tree_mask=mask, depth=depth, perm_k=perm, inv_perm_v=inverse(perm_v))
    out, amp, reach, _ = reference(cache, q, lens, perm, perm_v, mod, drafts=drafts, mask=mask, depth=depth)
    check(got, out, amp, reach)
    assert bool((got[1, max(1, T // 2):] == 0).all())          # rows behind a sequence's drafts
    assert B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [4, 40])
@pytest.mark.parametrize("kind", ["cap", "bias", "window", "window1", "first", "prefix", "all"])
def test_tree_attn_modified_scores(kind, T, dtype):
    cache, perm, perm_v, q = case(11, 3, 2, 2, 1024, T, dtype, 4, 32)
    lens, drafts = i32(900, 260, 0), i32(T, T, T)
    mask, depth = trees(3, T, drafts, 6)
    slopes = torch.tensor([0.5, 0.03, 0.0, 0.01], device="cuda")
    mod = {"cap": B.ScoreMod(softcap=3.0), "bias": B.ScoreMod(slopes=slopes), "window": B.ScoreMod(window=200),
           "window1": B.ScoreMod(window=1), "first": B.ScoreMod(first=i32(850, 260, 5)),
           "prefix": B.ScoreMod(window=30, prefix=i32(130, 1, 0)),
           "all": B.ScoreMod(softcap=5.0, slopes=slopes, window=500, first=i32(600, 2, 0), prefix=i32(3, 0, 9))}[kind]
    got = B.tree_attn(cache, q, lens, draft_lens=drafts, tree_mask=mask, depth=depth, perm_k=perm,
                      inv_perm_v=inverse(perm_v), mod=mod, softmax_scale=0.11)
    out, amp, reach, _ = reference(cache, q, lens, perm, perm_v, mod, scale=0.11, drafts=drafts, mask=mask, depth=depth)
    check(got, out, amp, reach, cap=mod.softcap)


@pytest.mark.gpu
def test_tree_attn_chain_is_the_default_and_empty_masks_give_zeros():
    T = 9
    cache, perm, perm_v, q = case(21, 2, 2, 2, 320, T, torch.float32, 4, 32)
    lens, drafts = i32(200, 17), i32(T, T)
    mask, depth = trees(2, T, drafts, 0, chain=True)
    kw = dict(perm_k=perm, inv_perm_v=inverse(perm_v))
    full = B.tree_attn(cache, q, lens, draft_lens=drafts, tree_mask=mask, depth=depth, **kw)
    assert torch.equal(full, B.tree_attn(cache, q, lens, **kw))
    none = torch.zeros_like(mask)
    got = B.tree_attn(cache, q, i32(0, 0), tree_mask=none, depth=depth, **kw)
    assert bool((got == 0).all())
    hidden = B.ScoreMod(first=i32(10 ** 9, 17))                 # the context hidden, drafted tokens not
    got = B.tree_attn(cache, q, lens, tree_mask=none, mod=hidden, **kw)
    assert bool((got == 0).all())
    assert B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,bits", [(torch.bfloat16, 4), (torch.float32, 8), (torch.bfloat16, 6)])
def test_tree_attn_equals_tokens_one_by_one(dtype, bits):
    """A chain of drafted tokens gives what the single-token form gives for each prefix of it."""
    T, S = 6, 700
    cache, perm, perm_v, q = case(31, 2, 2, 4, 720, T, dtype, bits, 32)
    lens = i32(S, 300)
    kw = dict(perm_k=perm, inv_perm_v=inverse(perm_v))
    mod = B.ScoreMod(softcap=8.0, slopes=torch.linspace(0.0, 0.05, 8, device="cuda"), window=257, prefix=i32(5, 5))
    tree = B.tree_attn(cache, q, lens, mod=mod, **kw).double()
    for i in range(T):
        one = B.decode_attn_mod(cache, q[:, i].contiguous(), lens + i + 1, mod, **kw)
        ref = reference(cache, q[:, i:i + 1].contiguous(), lens + i + 1, perm, perm_v, mod)
        check(one[:, None], *ref[:3], cap=8.0)
        check(tree[:, i:i + 1].to(dtype), *ref[:3], cap=8.0)


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [2.0 ** 100, 2.0 ** -100])
def test_large_and_small_cached_values(scale):
    """Values far from one: nothing leaves its range inside the kernels (queries are scaled against the keys)."""
    cache, perm, perm_v = make_cache(1, 2, 160, 4, 32, 3, scale=scale)
    q = (torch.randn(1, 3, 4, D, generator=torch.Generator().manual_seed(1)) / scale).cuda()
    lens = i32(150)
    got = B.tree_attn(cache, q, lens, perm_k=perm, inv_perm_v=inverse(perm_v))
    mask, depth = trees(1, 3, None, 0, chain=True)
    out, amp, reach, _ = reference(cache, q, lens, perm, perm_v, B.ScoreMod(), drafts=i32(3), mask=mask, depth=depth)
    check(got / scale, out / scale, amp / scale, reach)


@pytest.mark.gpu
def test_tree_attn_rows_past_the_end_do_not_matter():
    """Bytes of rows that no query sees may be anything, 255 exponents too."""
    cache, perm, perm_v, q = case(41, 2, 2, 2, 288, 5, torch.bfloat16, 4, 32)
    lens = i32(131, 40)
    mod = B.ScoreMod(window=64, prefix=i32(2, 2))
    want = B.tree_attn(cache, q, lens, mod=mod, perm_k=perm)
    mass = torch.zeros(2, 2, 288, device="cuda")
    one = B.decode_attn_mass(cache, q[:, 0].contiguous(), lens, mass, mod=mod, perm_k=perm)
    for b, n in enumerate((131, 40)):
        for plane in (cache.k_mant, cache.k_exp, cache.v_mant, cache.v_exp):
            plane[b, :, n + 5:] = 255
            plane[b, :, 2:max(2, n - 64)] = 255
    assert torch.equal(B.tree_attn(cache, q, lens, mod=mod, perm_k=perm), want)
    again = torch.zeros_like(mass)
    assert torch.equal(B.decode_attn_mass(cache, q[:, 0].contiguous(), lens, again, mod=mod, perm_k=perm), one)
    assert torch.equal(again, mass)


@pytest.mark.gpu
def test_lengths_outside_the_cache_are_clamped_and_flagged():
    cache, perm, perm_v, q = case(51, 2, 1, 1, 64, 4, torch.float32, 4, 32)
    got = B.tree_attn(cache, q, i32(62, -3), perm_k=perm, inv_perm_v=inverse(perm_v))
    assert B.device_status() == B.FLAG_POSITION
    mask, depth = trees(2, 4, None, 0, chain=True)
    out, amp, reach, _ = reference(cache, q, i32(62, 0), perm, perm_v, B.ScoreMod(), drafts=i32(4, 4), mask=mask, depth=depth)
    check(got, out, amp, reach)                                  # two drafted rows exist, the other queries give zeros
    assert bool((got[0, 2:] == 0).all())
    got = B.decode_attn_mod(cache, q[:, 0].contiguous(), i32(1000, 0), B.ScoreMod(), perm_k=perm, inv_perm_v=inverse(perm_v))
    assert B.device_status() == B.FLAG_POSITION
    out, amp, reach, _ = reference(cache, q[:, :1].contiguous(), i32(64, 0), perm, perm_v, B.ScoreMod())
    check(got[:, None], out, amp, reach)
    assert bool((got[1] == 0).all())


@pytest.mark.gpu
def test_non_finite_queries_stay_in_their_rows():
    cache, perm, perm_v, q = case(61, 1, 1, 1, 256, 6, torch.bfloat16, 4, 32)
    clean = B.tree_attn(cache, q, i32(200), perm_k=perm)
    q2 = q.clone()
    q2[0, 2, 0, 9] = float("nan")
    q2[0, 4, 0, 1] = float("inf")
    got = B.tree_attn(cache, q2, i32(200), perm_k=perm)
    keep = [0, 1, 3, 5]
    assert torch.equal(got[:, keep], clean[:, keep])
    assert bool(torch.isnan(got[0, 2]).all())


# ----------------------------------------------------------------------------------------------- single tokens
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits,block", FMT)
@pytest.mark.parametrize("group", [1, 4, 7, 8])
def test_decode_attn_mod_formats(bits, block, group, dtype):
    cache, perm, perm_v, q = case(group, 4, 2, group, 1104, 1, dtype, bits, block)
    lens = i32(1103, 1, 0, 513)
    mod = B.ScoreMod(softcap=6.0, window=400, prefix=i32(140, 3, 3, 0), first=i32(0, 0, 0, 300),
                     slopes=torch.linspace(0.0, 0.02, 2 * group, device="cuda"))
    got = B.decode_attn_mod(cache, q[:, 0].contiguous(), lens, mod, perm_k=perm, inv_perm_v=inverse(perm_v))
    out, amp, reach, _ = reference(cache, q, lens, perm, perm_v, mod)
    check(got[:, None], out, amp, reach, cap=6.0)
    assert bool((got[2] == 0).all())


@pytest.mark.gpu
def test_decode_attn_mod_without_mod_is_decode_attn():
    cache, perm, perm_v, q = case(71, 2, 4, 2, 528, 1, torch.float32, 4, 32)
    lens = i32(528, 77)
    a = B.decode_attn_mod(cache, q[:, 0].contiguous(), lens, None, perm_k=perm)
    b = B.decode_attn(cache, q[:, 0].contiguous(), lens, perm_k=perm)
    assert float(((a - b).abs().amax(-1) / b.abs().amax(-1)).max()) <= 2e-3      # the bound of decode_attn itself


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits,block", [(4, 32), (6, 16), (8, 64)])
@pytest.mark.parametrize("group,window", [(1, 0), (3, 0), (8, 150)])
def test_decode_attn_mass(bits, block, group, window, dtype):
    cache, perm, perm_v, q = case(81 + group, 3, 2, group, 912, 1, dtype, bits, block)
    lens = i32(901, 0, 130)
    mod = B.ScoreMod(softcap=10.0, window=window, prefix=i32(7, 7, 7) if window else None)
    mass = torch.rand(3, 2, 912, device="cuda")
    before = mass.clone()
    got = B.decode_attn_mass(cache, q[:, 0].contiguous(), lens, mass, mod=mod, perm_k=perm, inv_perm_v=inverse(perm_v))
    out, amp, reach, w = reference(cache, q, lens, perm, perm_v, mod)
    check(got[:, None], out, amp, reach, cap=10.0)
    # a weight is off by twice the score error (its own and the sum's), 2^-20 for exp2 and the sum, a rounding per addition
    d = 24 * 2.0 ** -23 * float(reach.max()) + 10.0 * 2.0 ** -21
    err = (mass.double() - before.double() - w).abs()
    assert bool((err <= w * (2 * d + 2.0 ** -19) + (group + 1) * 2.0 ** -24 * (mass.double() + w) + 1e-30).all())
    assert torch.equal(mass[w == 0], before[w == 0])             # nothing else is touched
    assert torch.equal(got, B.decode_attn_mod(cache, q[:, 0].contiguous(), lens, mod, perm_k=perm, inv_perm_v=inverse(perm_v)))


# ----------------------------------------------------------------------------------------------- many tiles, many blocks
@pytest.mark.gpu
@pytest.mark.parametrize("batch,heads,group,T,S,dtype,bits", [
    (1, 1, 1, 1, 40000, torch.bfloat16, 4),           # one pair over every thread block
    (1, 2, 4, 16, 12000, torch.bfloat16, 4),          # 64 rows
    (2, 3, 2, 20, 3000, torch.bfloat16, 8),           # 40 rows, ranges that begin and end inside pairs
    (37, 5, 1, 2, 260, torch.bfloat16, 6),            # more pairs than blocks
    (3, 2, 8, 30, 500, torch.float32, 4),             # 240 fp32 rows in tiles of 16
    (2, 1, 8, 64, 900, torch.bfloat16, 4)])           # 512 rows in tiles of 64
def test_many_tiles(batch, heads, group, T, S, dtype, bits):
    """Work cut over many blocks and partials, against fp64 on the GPU by matrix products."""
    max_seq = (S + T + 15) // 16 * 16
    cache, perm, perm_v, q = case(91, batch, heads, group, max_seq, T, dtype, bits, 32)
    lens = torch.tensor([max(0, S - 117 * b) for b in range(batch)], dtype=torch.int32, device="cuda")
    got = B.tree_attn(cache, q, lens, perm_k=perm, inv_perm_v=inverse(perm_v))
    k = B.dequant_all(cache, "k", max_seq, perm=perm).double()
    v = B.dequant_all(cache, "v", max_seq, perm=perm_v).double()
    out, amp = torch.zeros_like(got, dtype=torch.float64), torch.zeros_like(got, dtype=torch.float64)
    reach = torch.zeros(got.shape[:-1], dtype=torch.float64, device="cuda")
    t = torch.arange(max_seq, device="cuda")
    for b in range(batch):
        see = t <= lens[b] + torch.arange(T, device="cuda")[:, None]
        for h in range(heads):
            for qi in range(h * group, (h + 1) * group):
                x = (q[b, :, qi].double() @ k[b, :, h].T) / math.sqrt(D)
                p = torch.softmax(x.masked_fill(~see, -math.inf), -1)
                out[b, :, qi], amp[b, :, qi] = p @ v[b, :, h], p @ v[b, :, h].abs()
                reach[b, :, qi] = (q[b, :, qi].double().abs() @ k[b, :, h].abs().T).amax(-1) / math.sqrt(D)
    check(got, out, amp, reach)
    assert torch.equal(got, B.tree_attn(cache, q, lens, perm_k=perm, inv_perm_v=inverse(perm_v)))
    assert B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("batch,T,dtype", [(300, 1, torch.bfloat16), (1024, 2, torch.float32), (260, 10, torch.bfloat16)])
def test_many_sequences(batch, T, dtype):
    """More sequences than a block has threads, a third of them empty, the first and the last among those."""
    cache, perm, perm_v, q = case(141, batch, 1, 1, 48, T, dtype, 4, 32)
    rng = np.random.default_rng(2)
    n = rng.integers(0, 48 - T + 1, batch)
    n[rng.random(batch) < 0.3] = 0
    n[0] = n[-1] = 0
    drafts = rng.integers(0, T + 1, batch)
    drafts[[0, -1]] = 0
    lens, drafts = (torch.from_numpy(x.astype(np.int32)).cuda() for x in (n, drafts))
    mask, depth = trees(batch, T, drafts, 9)
    if T == 1:
        got = B.decode_attn_mod(cache, q[:, 0].contiguous(), lens, None, perm_k=perm, inv_perm_v=inverse(perm_v))[:, None]
        ref = reference(cache, q, lens, perm, perm_v, B.ScoreMod())
    else:
        got = B.tree_attn(cache, q, lens, draft_lens=drafts, tree_mask=mask, depth=depth, perm_k=perm, inv_perm_v=inverse(perm_v))
        ref = reference(cache, q, lens, perm, perm_v, B.ScoreMod(), drafts=drafts, mask=mask, depth=depth)
    check(got, *ref[:3])
    assert bool((got[0] == 0).all()) and bool((got[-1] == 0).all()) and B.device_status() == 0


@pytest.mark.gpu
def test_streams_graphs_and_shared_arguments():
    """The same calls on two streams with a workspace each, and captured into a graph that is replayed on new data."""
    cache, perm, perm_v, q = case(101, 2, 4, 2, 640, 8, torch.bfloat16, 4, 32)
    lens = i32(600, 333)
    want = B.tree_attn(cache, q, lens, perm_k=perm)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    ws = [torch.empty(B.attn_workspace_bytes(cache.fmt, 8, 8), dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = []
    for _ in range(6):
        for s, w in ((s1, ws[0]), (s2, ws[1])):
            with torch.cuda.stream(s):
                outs.append(B.tree_attn(cache, q, lens, perm_k=perm, workspace=w))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)

    mass = torch.zeros(2, 4, 640, device="cuda")
    q1 = q[:, 0].contiguous()
    out = torch.empty_like(q1)
    w = torch.empty(B.attn_workspace_bytes(cache.fmt, 8, 1, True), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        B.decode_attn_mass(cache, q1, lens, mass, perm_k=perm, out=out, workspace=w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.decode_attn_mass(cache, q1, lens, mass, perm_k=perm, out=out, workspace=w)
    mass.zero_()
    q1.copy_(q[:, 5])
    lens.copy_(i32(20, 500))
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    again = torch.zeros_like(mass)
    for _ in range(2):
        ref = B.decode_attn_mass(cache, q1, lens, again, perm_k=perm)
    assert torch.equal(out, ref) and torch.equal(mass, again)


# ----------------------------------------------------------------------------------------------- eviction, row moves
def plain_kept(mass, n, budget, sink, recent):
    if n <= budget:
        return np.arange(n)
    mid = np.arange(sink, n - recent)
    key = np.where(np.isnan(mass[mid]), -np.inf, mass[mid].astype(np.float64))
    nan_last = np.isnan(mass[mid])
    order = np.lexsort((mid, nan_last, -key))
    best = mid[order[:budget - sink - recent]]
    return np.concatenate([np.arange(sink), np.sort(best), np.arange(n - recent, n)]).astype(np.int64)


def planes(cache):
    return [cache.k_mant, cache.k_exp, cache.v_mant, cache.v_exp]


def weights_for(kind, shape, seed):
    g = torch.Generator().manual_seed(seed)
    m = torch.rand(shape, generator=g) ** 4
    if kind == "ties":
        m = torch.round(m * 8) / 8
    if kind == "equal":
        m = torch.full(shape, 0.25)
    if kind == "odd":
        m = torch.randn(shape, generator=g)
        m[..., ::7] = 0.0
        m[..., 1::7] = -0.0
        m[..., 2::11] = float("nan")
        m[..., 3::13] = float("inf")
        m[..., 4::17] = -float("inf")
    return m.cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("bits,block", [(4, 32), (4, 16), (6, 32), (8, 128)])
@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "odd"])
@pytest.mark.parametrize("budget,sink,recent", [(100, 4, 30), (1, 0, 0), (1, 1, 0), (33, 0, 33), (260, 16, 0), (700, 5, 5)])
def test_evict(budget, sink, recent, kind, bits, block, in_place):
    Bn, H, S = 3, 2, 720
    cache, _, _ = make_cache(Bn, H, S, bits, block, 7)
    mass = weights_for(kind, (Bn, H, S), 9)
    lens = i32(711, 99, 0)
    src = [p.clone() for p in planes(cache)]
    m0 = mass.cpu().numpy().copy()
    if in_place:
        dst, dm = cache, mass
        kept, new = B.evict(cache, lens, mass, budget, sink, recent, new_lens=lens)
        assert new.data_ptr() == lens.data_ptr()
    else:
        rows = (budget + 31) // 16 * 16
        dst = B.Cache(Bn, H, D, rows, block, bits, fill=0x5A)
        dm = torch.full((Bn, H, rows), 9.0, device="cuda")
        kept, new = B.evict(cache, lens, mass, budget, sink, recent, dst=dst, dst_mass=dm)
        assert all(torch.equal(a, b) for a, b in zip(src, planes(cache))) and lens.tolist() == [711, 99, 0]
    assert new.tolist() == [min(n, budget) for n in (711, 99, 0)]
    for b, n in enumerate((711, 99, 0)):
        for h in range(H):
            want = plain_kept(m0[b, h], n, budget, sink, recent)
            c = len(want)
            assert kept[b, h].tolist() == want.tolist() + [-1] * (budget - c)
            w = torch.from_numpy(want).cuda()
            for p, q in zip(planes(dst), src):
                assert torch.equal(p[b, h, :c], q[b, h, w])
                if not in_place:
                    assert bool((p[b, h, c:] == 0x5A).all())
            assert np.array_equal(dm[b, h, :c].cpu().numpy(), m0[b, h, want], equal_nan=True)
            assert bool((dm[b, h, c:] == 0).all())
    assert B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("heads,S,budget", [(1, 70001, 5000), (3, 9000, 8990)])
def test_evict_long(heads, S, budget):
    max_seq = (S + 15) // 16 * 16
    cache, _, _ = make_cache(1, heads, max_seq, 4, 32, 17)
    mass = weights_for("ties", (1, heads, max_seq), 4) + weights_for("plain", (1, heads, max_seq), 5).round(decimals=3)
    m0 = mass.cpu().numpy().copy()
    src = [p.clone() for p in planes(cache)]
    kept, new = B.evict(cache, i32(S), mass, budget, 10, 100)
    for h in range(heads):
        want = plain_kept(m0[0, h], S, budget, 10, 100)
        assert np.array_equal(kept[0, h].cpu().numpy(), want)
        w = torch.from_numpy(want).cuda()
        for p, q in zip(planes(cache), src):
            assert torch.equal(p[0, h, :budget], q[0, h, w])
    assert new.tolist() == [budget]


@pytest.mark.gpu
@pytest.mark.parametrize("bits,block", [(4, 32), (6, 16), (8, 64)])
@pytest.mark.parametrize("per_head", [False, True])
def test_gather_rows(bits, block, per_head):
    Bn, H, S, T = 3, 2, 208, 64
    cache, _, _ = make_cache(Bn, H, S, bits, block, 27)
    rng = np.random.default_rng(1)
    base, count = [100, 0, 140], [13, 64, 0]
    idx = np.stack([np.stack([np.sort(rng.permutation(T)) if b != 0 else np.sort(rng.permutation(T)[:T]) for _ in range(H)])
                    for b in range(Bn)]).astype(np.int32)
    idx[0] = np.sort(np.stack([rng.permutation(T) for _ in range(H)]), axis=1)
    idx[0, :, :13] = np.sort(np.stack([rng.permutation(T)[:13] for _ in range(H)]), axis=1)
    if not per_head:
        idx[:, 1] = idx[:, 0]
    index = torch.from_numpy(idx if per_head else idx[:, 0].copy()).cuda()
    src = [p.clone() for p in planes(cache)]
    B.gather_rows(cache, index, i32(*count), i32(*base))
    other = B.Cache(Bn, H, D, 96, block, bits, fill=0x5A)
    mine = B.Cache.__new__(B.Cache)
    mine.fmt = cache.fmt
    mine.k_mant, mine.k_exp, mine.v_mant, mine.v_exp = src
    B.gather_rows(mine, index, i32(*count), i32(*base), dst=other, dst_base=i32(7, 32, 0))
    assert B.device_status() == 0
    for b in range(Bn):
        for h in range(H):
            rows = torch.from_numpy(idx[b, h, :count[b]].astype(np.int64) + base[b]).cuda()
            for p, o, q in zip(planes(cache), planes(other), src):
                want = q[b, h].clone()
                want[base[b]:base[b] + count[b]] = q[b, h, rows]
                assert torch.equal(p[b, h], want)
                to = torch.full_like(o[b, h], 0x5A)
                d0 = (7, 32, 0)[b]
                to[d0:d0 + count[b]] = q[b, h, rows]
                assert torch.equal(o[b, h], to)


@pytest.mark.gpu
def test_gather_rows_outside_the_cache_are_skipped():
    cache, _, _ = make_cache(1, 1, 32, 4, 32, 2)
    src = [p.clone() for p in planes(cache)]
    B.gather_rows(cache, torch.tensor([[0, 3, -1, 5]], dtype=torch.int32, device="cuda"), i32(4), i32(28))
    assert B.device_status() == B.FLAG_POSITION
    for p, q in zip(planes(cache), src):
        want = q.clone()
        want[0, 0, 29] = q[0, 0, 31]
        assert torch.equal(p, want)


@pytest.mark.gpu
def test_gather_rows_in_place_order():
    """In place: any order whose sources lie at or behind their destinations; others are skipped and flagged."""
    cache, _, _ = make_cache(1, 2, 448, 4, 32, 6)
    src = [p.clone() for p in planes(cache)]
    rng = np.random.default_rng(3)
    idx = np.minimum(np.arange(200) + rng.integers(0, 200, 200), 399).astype(np.int32)          # not ascending, some twice
    B.gather_rows(cache, torch.from_numpy(idx)[None].contiguous().cuda(), i32(200), i32(40))
    assert B.device_status() == 0
    for p, q in zip(planes(cache), src):
        want = q.clone()
        want[:, :, 40:240] = q[:, :, torch.from_numpy(idx).long().cuda() + 40]
        assert torch.equal(p, want)
    src = [p.clone() for p in planes(cache)]
    B.gather_rows(cache, i32(0, 1, 1, 7, 2)[None].contiguous(), i32(5))
    assert B.device_status() == B.FLAG_POSITION
    for p, q in zip(planes(cache), src):
        want = q.clone()
        want[:, :, 3] = q[:, :, 7]
        assert torch.equal(p, want)


@pytest.mark.gpu
def test_speculative_step_then_eviction():
    """As they are used together: draft a tree, score it, commit a branch, go on decoding with weights, evict, decode."""
    Bn, H, G, S, T = 2, 2, 2, 300, 7
    cache, perm, perm_v, q = case(111, Bn, H, G, 336, T, torch.float32, 4, 32)
    inv = inverse(perm_v)
    lens = i32(S, 250)
    g = torch.Generator().manual_seed(3)
    kd, vd = (torch.randn(Bn, T, H, D, generator=g).cuda() for _ in range(2))
    B.append(cache, kd, vd, lens, perm_k=perm, perm_v=perm_v)
    mask = torch.tensor([[1, 3, 5, 11, 21, 37, 75]] * Bn, dtype=torch.int64, device="cuda")
    depth = torch.tensor([[0, 1, 1, 2, 2, 2, 3]] * Bn, dtype=torch.int32, device="cuda")
    tree = B.tree_attn(cache, q, lens, tree_mask=mask, depth=depth, perm_k=perm, inv_perm_v=inv)
    # branch 0-1-3-6 accepted in the first sequence, 0-2 in the second
    index = torch.tensor([[0, 1, 3, 6], [0, 2, 0, 0]], dtype=torch.int32, device="cuda")
    B.gather_rows(cache, index, i32(4, 2), lens)
    # the tip's row of the tree is what decoding at its place gives
    tip = torch.stack([q[0, 6], q[1, 2]])
    mass = torch.zeros(Bn, H, 336, device="cuda")
    new = lens + i32(4, 2)
    one = B.decode_attn_mass(cache, tip, new, mass, perm_k=perm, inv_perm_v=inv)
    ref = reference(cache, tip[:, None].contiguous(), new, perm, perm_v, B.ScoreMod())
    check(one[:, None], *ref[:3])
    check(torch.stack([tree[0, 6], tree[1, 2]])[:, None].contiguous(), *ref[:3])
    assert torch.allclose(mass.sum(-1), torch.full((Bn, H), float(G), device="cuda"), atol=1e-4)
    # keep 64 rows, decode over them: attention over the kept rows only
    before = cache.k_mant.clone()
    kept, lens2 = B.evict(cache, new, mass, 64, 4, 16)
    assert lens2.tolist() == [64, 64]
    assert torch.equal(cache.k_mant[1, 1, :64], before[1, 1, kept[1, 1].long()])
    out = B.decode_attn(cache, tip, lens2, perm_k=perm, inv_perm_v=inv)
    mod = B.decode_attn_mod(cache, tip, lens2, None, perm_k=perm, inv_perm_v=inv)
    ref = reference(cache, tip[:, None].contiguous(), lens2, perm, perm_v, B.ScoreMod())
    check(mod[:, None], *ref[:3])
    assert float(((out.double() - ref[0][:, 0]).abs().amax(-1) / ref[0][:, 0].abs().amax(-1)).max()) <= 2e-3
    assert B.device_status() == 0


@pytest.mark.gpu
def test_rows_far_into_a_long_cache():
    """Offsets past 32 bits: the second head's rows lie 4 GB into the planes."""
    H, S, n = 2, (1 << 25) + (1 << 24), (1 << 25) + (1 << 24) - 37
    cache = B.Cache(1, H, D, S, 32, 4, fill=0x88)
    cache.k_exp.fill_(120)
    cache.v_exp.fill_(120)
    assert 2 * S * cache.fmt.row_m > 1 << 32
    small, _, _ = make_cache(1, H, 288, 4, 32, 31)
    # rows 0..287 of the small cache become rows n - 288 .. of the long one, and the last 200 of them come back
    index = torch.arange(288, dtype=torch.int32, device="cuda")[None].contiguous()
    B.gather_rows(small, index, i32(288), dst=cache, dst_base=i32(n - 288))
    back = B.Cache(1, H, D, 208, 32, 4, fill=0)
    B.gather_rows(cache, index[:, :200].contiguous(), i32(200), src_base=i32(n - 200), dst=back)
    for p, q in zip(planes(back), planes(small)):
        assert torch.equal(p[:, :, :200], q[:, :, 88:288])
    g = torch.Generator().manual_seed(8)
    for dtype in (torch.bfloat16, torch.float32):
        q = torch.randn(1, 2 * H, D, generator=g).to(dtype).cuda()
        got = B.decode_attn_mod(cache, q, i32(n), B.ScoreMod(window=200))
        ref = reference(back, q[:, None].contiguous(), i32(200), None, None, B.ScoreMod())
        check(got[:, None], *ref[:3])
    mass = torch.zeros(1, H, S, device="cuda")
    mass[0, 1, n - 300:n - 150] = 1.0
    mass[0, 0, 5] = 2.0
    kept, new = B.evict(cache, i32(n), mass, 208, 2, 50, dst=back, dst_mass=torch.empty(1, H, 208, device="cuda"))
    want = [list(range(2)) + [2, 3, 4, 5] + list(range(6, 158)) + list(range(n - 50, n)),
            list(range(2)) + list(range(2, 8)) + list(range(n - 300, n - 150)) + list(range(n - 50, n))]
    assert kept[0].tolist() == want and new.tolist() == [208]
    assert torch.equal(back.k_mant[0, 1, 158:], cache.k_mant[0, 1, n - 50:n])
    assert B.device_status() == 0


@pytest.mark.gpu
def test_calls_on_a_named_stream_own_their_buffers():
    """stream= with nothing else given: what the call allocates is not handed out again while it runs."""
    cache, perm, perm_v, q = case(121, 2, 4, 2, 2048, 8, torch.bfloat16, 4, 32)
    lens = i32(2000, 1333)
    want = B.tree_attn(cache, q, lens, perm_k=perm)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    outs = []
    for _ in range(20):
        outs.append(B.tree_attn(cache, q, lens, perm_k=perm, stream=side))
        torch.full((1 << 22,), 255, dtype=torch.uint8, device="cuda")          # would land in a freed workspace
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


@pytest.mark.gpu
def test_binding_refuses_what_the_kernels_could_not_read(monkeypatch):
    cache, perm, perm_v, q = case(131, 1, 2, 1, 64, 2, torch.bfloat16, 4, 32)
    mass = torch.zeros(1, 2, 64, device="cuda")
    before = B.launch_count()
    with pytest.raises(ValueError):
        B.tree_attn(cache, q, i32(40), perm_k=perm[:1].contiguous())
    with pytest.raises(ValueError):
        B.tree_attn(cache, q, i32(40), workspace=torch.empty(1 << 22, dtype=torch.uint8))
    with pytest.raises(ValueError):
        B.decode_attn_mass(cache, q[:, 0].contiguous(), i32(40), mass[:, :, :48].contiguous())
    with pytest.raises(ValueError):
        B.tree_attn(cache, q, i32(40, 40))
    here = torch.cuda.current_device()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: here + 1)
    for call in (lambda: B.tree_attn(cache, q, i32(40)), lambda: B.evict(cache, i32(40), mass, 16),
                 lambda: B.gather_rows(cache, i32(0, 1)[None].contiguous(), i32(2))):
        with pytest.raises(ValueError, match="current device"):
            call()
    assert B.launch_count() == before


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 6, 8])
def test_wide_and_narrow_calls_at_once(bits):
    """Narrow and wide trees, single tokens and weights on four streams at once, each as alone."""
    cache, perm, perm_v, q = case(151, 3, 4, 2, 1056, 20, torch.bfloat16, bits, 32)
    lens, q1, q3 = i32(1000, 0, 517), q[:, 0].contiguous(), q[:, :3].contiguous()
    mod = B.ScoreMod(softcap=20.0, window=700)
    ws = [torch.empty(B.attn_workspace_bytes(cache.fmt, 8, 20, True), dtype=torch.uint8, device="cuda") for _ in range(4)]
    mass = [torch.zeros(3, 4, 1056, device="cuda") for _ in range(2)]
    calls = [lambda m: B.tree_attn(cache, q, lens, perm_k=perm, workspace=ws[0]),
             lambda m: B.tree_attn(cache, q3, lens, perm_k=perm, mod=mod, workspace=ws[1]),
             lambda m: B.decode_attn_mod(cache, q1.float(), lens, mod, perm_k=perm, workspace=ws[2]),
             lambda m: B.decode_attn_mass(cache, q1, lens, m, perm_k=perm, workspace=ws[3])]
    want = [c(mass[0]) for c in calls]
    for _ in range(4):
        calls[3](mass[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = []
    for _ in range(5):
        for s, c in zip(streams, calls):
            with torch.cuda.stream(s):
                got.append(c(mass[1]))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i % 4]) for i, g in enumerate(got)) and torch.equal(mass[0], mass[1])
    assert B.device_status() == 0


@pytest.mark.gpu
def test_whole_step_in_a_graph():
    """Draft, score, commit, decode with weights and evict in place, captured once and replayed on restored caches."""
    Bn, H, G, S, T = 2, 4, 2, 400, 12
    cache, perm, perm_v, q = case(161, Bn, H, G, 432, T, torch.bfloat16, 4, 32)
    g = torch.Generator().manual_seed(4)
    kd, vd = (torch.randn(Bn, T, H, D, generator=g).cuda() for _ in range(2))
    mask, depth = trees(Bn, T, None, 3)
    index = torch.tensor([[0, 2, 5, 11], [1, 3, 0, 0]], dtype=torch.int32, device="cuda")
    count, lens = i32(4, 2), i32(S, 250)
    mass, new, kept = torch.zeros(Bn, H, 432, device="cuda"), i32(0, 0), torch.empty(Bn, H, 128, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.attn_workspace_bytes(cache.fmt, H * G, T, True), dtype=torch.uint8, device="cuda")
    tree, one, tip = torch.empty_like(q), torch.empty_like(q[:, 0].contiguous()), q[:, 0].contiguous()

    def step():
        B.append(cache, kd, vd, lens, perm_k=perm, perm_v=perm_v)
        B.tree_attn(cache, q, lens, tree_mask=mask, depth=depth, perm_k=perm, out=tree, workspace=ws)
        B.gather_rows(cache, index, count, lens)
        lens.add_(count)
        B.decode_attn_mass(cache, tip, lens, mass, perm_k=perm, out=one, workspace=ws)
        B.evict(cache, lens, mass, 128, 4, 16, new_lens=lens, kept=kept)

    state = planes(cache) + [mass, lens, kept, tree, one]
    start = [x.clone() for x in state]

    def restore():
        for x, y in zip(state, start):
            x.copy_(y)

    step()
    torch.cuda.synchronize()
    want = [x.clone() for x in state]
    restore()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        restore()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(state, want))
    assert lens.tolist() == [128, 128] and B.device_status() == 0


# ----------------------------------------------------------------------------------------------- refusals (CPU)
def test_workspace_sizes():
    f = B.Format(2, 4, 128, 64, 32, 4)
    assert B.attn_workspace_bytes(f, 6, 1) == 0 and B.attn_workspace_bytes(f, 8, 0) == 0
    one, tree, mass = B.attn_workspace_bytes(f, 8, 1), B.attn_workspace_bytes(f, 8, 64), B.attn_workspace_bytes(f, 8, 1, True)
    assert 0 < one < tree and mass >= one + 2 * 8 * 64 * 4
    assert B.attn_workspace_bytes(B.Format(2, 4, 64, 64, 32, 4), 8, 1) == 0


def test_attention_refusals():
    L, vp = B.lib(), C.c_void_p
    f = B.Format(1, 2, 128, 32, 32, 4)
    cs = B.CacheStruct(f, 0x1000, 0x2000, 0x3000, 0x4000)
    need = B.attn_workspace_bytes(f, 4, 64)
    before = B.launch_count()

    def tree(cache=cs, q=vp(16), dt=1, hq=4, T=8, ctx=vp(16), mask=vp(16), scale=0.0, mod=None, out=vp(16), ws=vp(16), n=need):
        return L.kvbfp_tree_attn(None if cache is None else C.byref(cache), q, dt, hq, T, ctx, None, mask, None, None, None,
                                 scale, None if mod is None else C.byref(mod), out, ws, n, None)

    bad = [dict(cache=None), dict(q=None), dict(out=None), dict(ctx=None), dict(dt=2), dict(hq=3), dict(hq=0), dict(T=0),
           dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
           dict(mod=B.ScoreModStruct(-1.0, 0, None, None, None)), dict(mod=B.ScoreModStruct(float("nan"), 0, None, None, None)),
           dict(mod=B.ScoreModStruct(float("inf"), 0, None, None, None)), dict(mod=B.ScoreModStruct(0.0, -1, None, None, None)),
           dict(mod=B.ScoreModStruct(1e-21, 0, None, None, None)),
           dict(cache=B.CacheStruct(f, 0x1000, 0x2000, 0x3000, None))]
    for kw in bad:
        assert tree(**kw) == B.ERR_INVALID_ARG, kw
    for kw in (dict(hq=18), dict(T=65), dict(cache=B.CacheStruct(B.Format(1025, 2, 128, 32, 32, 4), 16, 16, 16, 16)),
               dict(cache=B.CacheStruct(B.Format(1, 2, 64, 32, 32, 4), 16, 16, 16, 16))):
        assert tree(**kw) == B.ERR_UNSUPPORTED, kw
    for kw in (dict(q=vp(8)), dict(out=vp(24)), dict(ws=vp(8)), dict(mask=vp(8))):
        assert tree(**kw) == B.ERR_ALIGNMENT, kw
    for kw in (dict(ws=None), dict(n=B.attn_workspace_bytes(f, 4, 8) - 1)):
        assert tree(**kw) == B.ERR_WORKSPACE, kw
    mass = lambda m, n: L.kvbfp_decode_attn_mass(C.byref(cs), vp(16), 1, 4, vp(16), None, None, 0.0, None, m, vp(16), vp(16), n, None)
    assert mass(None, 1 << 30) == B.ERR_INVALID_ARG
    assert mass(vp(8), 1 << 30) == B.ERR_ALIGNMENT
    assert mass(vp(16), B.attn_workspace_bytes(f, 4, 1)) == B.ERR_WORKSPACE
    assert L.kvbfp_decode_attn_mod(C.byref(cs), vp(16), 1, 4, None, None, None, 0.0, None, vp(16), vp(16), 1 << 30, None) == B.ERR_INVALID_ARG
    assert B.launch_count() == before


def test_eviction_refusals():
    L, vp = B.lib(), C.c_void_p
    f, small = B.Format(1, 2, 128, 64, 32, 4), B.Format(1, 2, 128, 32, 32, 4)
    src = B.CacheStruct(f, 0x100000, 0x200000, 0x300000, 0x400000)
    dst = B.CacheStruct(small, 0x500000, 0x600000, 0x700000, 0x800000)
    before = B.launch_count()

    def evict(s=src, d=dst, lens=vp(16), mass=vp(0x10000), budget=16, sink=4, recent=4, dm=vp(0x20000), new=vp(16), kept=vp(16)):
        return L.kvbfp_evict(C.byref(s), lens, mass, budget, sink, recent, C.byref(d), dm, new, kept, None)

    for kw in (dict(lens=None), dict(mass=None), dict(dm=None), dict(new=None), dict(kept=None), dict(budget=0),
               dict(sink=-1), dict(recent=-1), dict(sink=10, recent=7), dict(sink=17),
               dict(dm=vp(0x10000)),                                                        # another cache, the same masses
               dict(dm=vp(0x10100)),                                                        # masses that overlap
               dict(d=src),                                                                 # in place, other masses
               dict(d=B.CacheStruct(f, 0x100000, 0x200000, 0x300000, 0x500000)),            # some planes shared
               dict(d=B.CacheStruct(small, 0x100400, 0x600000, 0x700000, 0x800000)),        # planes that overlap
               dict(d=B.CacheStruct(B.Format(2, 2, 128, 32, 32, 4), 16, 32, 48, 64)),
               dict(d=B.CacheStruct(B.Format(1, 2, 128, 32, 16, 4), 16, 32, 48, 64)),
               dict(d=B.CacheStruct(B.Format(1, 2, 128, 32, 32, 8), 16, 32, 48, 64))):
        assert evict(**kw) == B.ERR_INVALID_ARG, kw
    assert evict(budget=33) == B.ERR_CAPACITY
    assert evict(mass=vp(0x10008)) == B.ERR_ALIGNMENT
    assert evict(d=B.CacheStruct(small, 0x500008, 0x600000, 0x700000, 0x800000)) == B.ERR_ALIGNMENT
    move = lambda idx=vp(16), heads=1, n=4, count=vp(16): L.kvbfp_gather_rows(C.byref(src), C.byref(dst), idx, heads, n, count, None, None, None)
    for kw in (dict(idx=None), dict(heads=3), dict(heads=0), dict(n=0), dict(count=None)):
        assert move(**kw) == B.ERR_INVALID_ARG, kw
    assert B.launch_count() == before


def test_binding_checks_shapes():
    t = torch.zeros(4)
    with pytest.raises(ValueError):
        B.ScoreMod(slopes=t)                                     # not on the device
    with pytest.raises(ValueError):
        B._sized("x", t, (5,))
    assert B._sized("x", None, (5,)) is None
