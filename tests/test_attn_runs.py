"""Attention over the packed cache where every worker of the kernels has several tiles and several runs (tiles of one
sequence, head and row tile), against fp64 matrix products on the dequantised cache."""
import ctypes as C
import math
import os

import numpy as np
import pytest
import torch

from paper_2403_20137_b200 import binding as B, build
from test_attn_ops import D, check, i32, inverse, trees


# ----------------------------------------------------------------------------------------------- helpers
def long_case(seed, batch, heads, group, max_seq, T, dtype, bits, block, empty=0.1):
    """Ragged sequences, made on the GPU; keys grow along the sequence, so that the running maxima keep rising."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    grow = (0.2 + 2.8 * torch.arange(max_seq, device="cuda") / max_seq)[None, :, None, None]
    k = torch.randn(batch, max_seq, heads, D, generator=g, device="cuda") * grow
    v = torch.randn(batch, max_seq, heads, D, generator=g, device="cuda")
    perm, perm_v = (torch.rand(heads, D, generator=g, device="cuda").argsort(-1).to(torch.int32).contiguous() for _ in range(2))
    cache = B.Cache(batch, heads, D, max_seq, block, bits)
    B.append(cache, k, v, torch.zeros(batch, dtype=torch.int32, device="cuda"), perm_k=perm, perm_v=perm_v)
    q = torch.randn(batch, T, heads * group, D, generator=g, device="cuda").to(dtype)
    lens = rng.integers(1, max_seq - T + 1, batch)
    lens[rng.random(batch) < empty] = 0
    lens[batch // 2] = max_seq - T
    return cache, perm, perm_v, q, torch.from_numpy(lens.astype(np.int32)).cuda()


def wide_reference(cache, q, lens, perm, perm_v, mod, scale=0.0, drafts=None, mask=None, depth=None, weights=None):
    """-> out, the sum of p|v| per output, the largest sum of |q k| scale of a row's visible tokens; all fp64.
    q [B, T, Hq, D]; drafts None: a single token at lens - 1.  `weights` [B, H, max_seq]: the softmax weights are added."""
    f = cache.fmt
    Bn, T, Hq, _ = q.shape
    H, G = f.n_kv_heads, Hq // f.n_kv_heads
    scale = scale or 1.0 / math.sqrt(D)
    k, v = B.dequant_all(cache, "k", f.max_seq, perm=perm), B.dequant_all(cache, "v", f.max_seq, perm=perm_v)
    out = torch.zeros(Bn, T, Hq, D, dtype=torch.float64, device="cuda")
    amp, reach = torch.zeros_like(out), torch.zeros(Bn, T, Hq, dtype=torch.float64, device="cuda")
    back = lambda x: x.reshape(H, T, G, -1).transpose(0, 1).reshape(T, Hq, -1)
    for b, n in enumerate(lens.tolist()):
        nd = 0 if drafts is None else int(drafts[b])
        m = n + nd
        if m == 0 or (drafts is not None and nd == 0):
            continue
        kp = torch.arange(m, device="cuda")
        pos = torch.tensor([n - 1], device="cuda") if drafts is None else n + depth[b].long()
        if nd:
            kp[n:] = n + depth[b, :nd].long()
        near = (pos[:, None] - kp < mod.window) if mod.window else torch.ones(T, m, dtype=torch.bool, device="cuda")
        see = near.clone()
        if mod.first is not None:
            see[:, :n] &= kp[:n] >= min(max(int(mod.first[b]), 0), n)
        if mod.prefix is not None:
            see[:, :n] |= kp[:n] < min(max(int(mod.prefix[b]), 0), n)
        if nd:
            see[:, n:] = ((mask[b][:, None] >> torch.arange(nd, device="cuda")) & 1).bool() & near[:, n:]
            see[nd:] = False
        kb, vb = (x[b, :m].double().transpose(0, 1) for x in (k, v))                              # [H, m, D]
        qb = q[b].double().reshape(T, H, G, D).transpose(0, 1).reshape(H, T * G, D)
        seen = see.repeat_interleave(G, 0)[None]
        x = qb @ kb.transpose(1, 2) * scale
        r = (qb.abs() @ kb.abs().transpose(1, 2) * scale).masked_fill(~seen, 0.0).amax(-1)
        if mod.softcap:
            x = mod.softcap * torch.tanh(x / mod.softcap)
        if mod.slopes is not None:
            x = x - mod.slopes.double().reshape(H, 1, G, 1).expand(H, T, G, 1).reshape(H, T * G, 1) * (pos[:, None] - kp).repeat_interleave(G, 0)
        p = torch.softmax(x.masked_fill(~seen, -math.inf), -1).nan_to_num(0.0)
        out[b], amp[b], reach[b] = back(p @ vb), back(p @ vb.abs()), back(r[..., None])[..., 0]
        if weights is not None:
            weights[b, :, :m] += p.sum(1)
    return out, amp, reach


# ----------------------------------------------------------------------------------------------- runs after runs
@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 6, 8])
@pytest.mark.parametrize("T,group", [(16, 1), (8, 4), (33, 2)])
def test_value_order_of_each_head(T, group, bits):
    """Whole runs of one head after another, each head with a value order of its own: a run's results are in its own
    head's order (three widths of query rows)."""
    cache, perm, perm_v, q, lens = long_case(5, 128, 8, group, 640, T, torch.bfloat16, bits, 32)
    drafts = torch.full((128,), T, dtype=torch.int32, device="cuda")
    mask, depth = trees(128, T, drafts, 4)
    kw = dict(tree_mask=mask, depth=depth, perm_k=perm, inv_perm_v=inverse(perm_v))
    got = B.tree_attn(cache, q, lens, **kw)
    check(got, *wide_reference(cache, q, lens, perm, perm_v, B.ScoreMod(), drafts=drafts, mask=mask, depth=depth))
    for _ in range(20):
        assert torch.equal(B.tree_attn(cache, q, lens, **kw), got)
    assert B.device_status() == 0


def test_channel_table_is_read_before_the_last_barrier_of_a_run():
    """The order that keeps two runs apart, in the source (a run too late by some hundred cycles would not show): the
    table is written before the first barrier of a run, so it has to be read before the last one."""
    with open(os.path.join(build.CSRC, "attn_umma.cuh")) as f:
        code = f.read()
    write, read = code.index("chan[a.inv_perm_v["), code.index("chan[slot_of]")
    end = code.index("c = cn;", read)
    sync = "named_sync(bar_id, 128);"
    assert code.index(sync, write) < read < code.rindex(sync, write, end)


ALL_FMT = [(bits, block) for bits in (4, 6, 8) for block in (16, 32, 64, 128)]


def check_long(got, out, amp, reach, max_seq, cap=0.0, lean=0.0):
    """The bound of check() with what it leaves out: a sum over S tokens has S / 16 steps of O that cut (2^-23 each) and
    S / 8 additions of weights (2^-24 each), S 2^-26 in all; a bias of up to `lean` is rounded four times; each of some
    ten moves of the reference rounds sums twice.  Weights of fp32 queries: three bf16 terms, 2^-24 and twice 2^-22 of exp2."""
    d = 24 * 2.0 ** -23 * reach + cap * 2.0 ** -21 + lean * 2.0 ** -22
    w = (2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -20) + max_seq * 2.0 ** -26 + 2.0 ** -19
    bound = amp * (2 * d[..., None] + w) * 1.01 + 2.0 ** (-8 if got.dtype == torch.bfloat16 else -24) * out.abs() * 1.01 + 1e-35
    worst = float(((got.double() - out).abs() / bound).max())
    assert bool(torch.isfinite(got).all()) and worst <= 1.0, f"error is {worst:.3g} of the bound"


def all_mods(batch, heads, lens, cap=25.0):
    """Cap, bias, window, document and prefix at once; -> the mod and the largest bias."""
    slopes = torch.linspace(0.0, 0.01, heads, device="cuda")
    mod = B.ScoreMod(softcap=cap, slopes=slopes, window=1500, first=(lens // 5).contiguous(),
                     prefix=torch.arange(batch, dtype=torch.int32, device="cuda") * 3)
    return mod, 0.01 * int(lens.max())


@pytest.mark.gpu
@pytest.mark.parametrize("modified", [False, True])
@pytest.mark.parametrize("bits,block", ALL_FMT)
@pytest.mark.parametrize("T,group", [(16, 1), (7, 4), (16, 4), (33, 2)])
def test_wide_trees_over_many_runs(T, group, bits, block, modified):
    """Every instance of the wide kernel with some ten tiles a worker: stages and barriers used over and over, sums
    carried over tiles while their references rise, runs that begin and end inside (sequence, head) pairs."""
    batch, heads, max_seq = 64, 8, 2080
    cache, perm, perm_v, q, lens = long_case(20 + T, batch, heads, group, max_seq, T, torch.bfloat16, bits, block)
    drafts = torch.tensor([max(0, T - b % 5) for b in range(batch)], dtype=torch.int32, device="cuda")
    mask, depth = trees(batch, T, drafts, 21)
    mod, lean = all_mods(batch, heads * group, lens) if modified else (B.ScoreMod(), 0.0)
    kw = dict(draft_lens=drafts, tree_mask=mask, depth=depth, perm_k=perm, inv_perm_v=inverse(perm_v), mod=mod)
    got = B.tree_attn(cache, q, lens, **kw)
    ref = wide_reference(cache, q, lens, perm, perm_v, mod, drafts=drafts, mask=mask, depth=depth)
    check_long(got, *ref, max_seq, cap=mod.softcap, lean=lean)
    for b in range(5):
        assert bool((got[b, max(0, T - b):] == 0).all())
    assert torch.equal(B.tree_attn(cache, q, lens, **kw), got) and B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("modified", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits,block", ALL_FMT)
@pytest.mark.parametrize("T,group", [(1, 1), (1, 5), (4, 2), (3, 4)])
def test_narrow_calls_over_many_runs(T, group, bits, block, dtype, modified):
    """The same for the narrow kernel (and 12 bf16 rows): single tokens and small trees, some ten tiles a warp."""
    batch, heads, max_seq = 64, 8, 4112 if bits == 4 else 2064
    cache, perm, perm_v, q, lens = long_case(30 + T, batch, heads, group, max_seq, T, dtype, bits, block)
    mod, lean = all_mods(batch, heads * group, lens) if modified else (B.ScoreMod(), 0.0)
    kw = dict(perm_k=perm, inv_perm_v=inverse(perm_v), mod=mod)
    if T == 1:
        call = lambda: B.decode_attn_mod(cache, q[:, 0].contiguous(), lens, **kw)[:, None]
        ref = wide_reference(cache, q, lens, perm, perm_v, mod)
    else:
        drafts = torch.full((batch,), T, dtype=torch.int32, device="cuda")
        mask, depth = trees(batch, T, drafts, 31)
        call = lambda: B.tree_attn(cache, q, lens, tree_mask=mask, depth=depth, **kw)
        ref = wide_reference(cache, q, lens, perm, perm_v, mod, drafts=drafts, mask=mask, depth=depth)
    got = call()
    check_long(got, *ref, max_seq, cap=mod.softcap, lean=lean)
    assert torch.equal(call(), got) and B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits,block", [(4, 32), (6, 16), (8, 128)])
@pytest.mark.parametrize("group,modified", [(1, False), (4, True)])
def test_weights_over_many_runs(bits, block, group, modified, dtype):
    """Attention weights where every warp has several tiles, added to what is there; their sum is the number of heads."""
    batch, heads, max_seq = 64, 8, 4112 if bits == 4 else 2064
    cache, perm, perm_v, q, lens = long_case(40, batch, heads, group, max_seq, 1, dtype, bits, block)
    mod, lean = all_mods(batch, heads * group, lens) if modified else (B.ScoreMod(), 0.0)
    mass = torch.rand(batch, heads, max_seq, device="cuda")
    before, w = mass.clone(), torch.zeros(batch, heads, max_seq, dtype=torch.float64, device="cuda")
    q1 = q[:, 0].contiguous()
    got = B.decode_attn_mass(cache, q1, lens, mass, mod=mod, perm_k=perm, inv_perm_v=inverse(perm_v))
    ref = wide_reference(cache, q, lens, perm, perm_v, mod, weights=w)
    check_long(got[:, None], *ref, max_seq, cap=mod.softcap, lean=lean)
    assert torch.equal(got, B.decode_attn_mod(cache, q1, lens, mod, perm_k=perm, inv_perm_v=inverse(perm_v)))
    # a weight: twice the score's error, exp2 twice, the sum (S 2^-27 and the moves of the reference); a rounding per addition
    d = 24 * 2.0 ** -23 * float(ref[2].max()) + mod.softcap * 2.0 ** -21 + lean * 2.0 ** -22
    bound = w * (2 * d + 2.0 ** -19 + max_seq * 2.0 ** -27) + (group + 1) * 2.0 ** -24 * (mass.double() + w) + 1e-30
    assert bool(((mass.double() - before.double() - w).abs() <= bound).all())
    assert torch.equal(mass[w == 0], before[w == 0]) and B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("T,group", [(12, 1), (10, 2), (20, 2), (17, 4)])
def test_non_finite_queries_of_wide_trees_stay_in_their_rows(T, group):
    """More than eight rows: each width of the wide kernel."""
    cache, perm, perm_v, q, _ = long_case(50, 2, 2, group, 416, T, torch.bfloat16, 4, 32)
    lens = i32(380, 200)
    clean = B.tree_attn(cache, q, lens, perm_k=perm, inv_perm_v=inverse(perm_v))
    bad = q.clone()
    bad[0, 3, 0, 17] = float("nan")
    bad[1, T - 1, 2 * group - 1, 90] = float("inf")
    bad[1, 5, 0, 2] = -float("inf")
    got = B.tree_attn(cache, bad, lens, perm_k=perm, inv_perm_v=inverse(perm_v))
    rows = torch.zeros(2, T, 2 * group, dtype=torch.bool)
    rows[0, 3, 0] = rows[1, T - 1, 2 * group - 1] = rows[1, 5, 0] = True
    assert torch.equal(got[~rows], clean[~rows]) and bool(torch.isnan(got[rows]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits,block", [(4, 32), (6, 16), (6, 128), (8, 32)])
@pytest.mark.parametrize("T,group", [(3, 1), (12, 1), (9, 3), (20, 3)])
@pytest.mark.parametrize("power", [113, -95])
def test_cached_magnitudes_at_the_ends_of_the_range(power, T, group, bits, block, dtype):
    """Keys and values around 2^113 (loud channels near 2^117) and 2^-95, each width; the scale makes up for the keys."""
    g = torch.Generator(device="cuda").manual_seed(60 + T)
    s = 2.0 ** power
    k, v = (torch.randn(2, 304, 2, D, generator=g, device="cuda") * s for _ in range(2))
    k[..., [3, 77, 120]] *= 3.0
    cache = B.Cache(2, 2, D, 304, block, bits)
    B.append(cache, k, v, i32(0, 0))
    q = torch.randn(2, T, 2 * group, D, generator=g, device="cuda").to(dtype)
    lens, drafts, scale = i32(280, 130), i32(T, T), 2.0 ** -power / math.sqrt(D)
    mask, depth = trees(2, T, drafts, 61)
    got = B.tree_attn(cache, q, lens, tree_mask=mask, depth=depth, softmax_scale=scale)
    out, amp, reach = wide_reference(cache, q, lens, None, None, B.ScoreMod(), scale=scale, drafts=drafts, mask=mask, depth=depth)
    check(got / s, out / s, amp / s, reach)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cap", [0.0, 1e6])
@pytest.mark.parametrize("T", [3, 12, 40])
@pytest.mark.parametrize("power,scale", [(100, 2.0 ** 60), (0, 3e38)])
def test_scores_of_zero_stay_zero_under_any_scale(power, scale, T, cap, dtype):
    """The scale times the cached magnitudes may leave the fp32 range: rows of zeros weigh all they see alike."""
    g = torch.Generator(device="cuda").manual_seed(90)
    k, v = (torch.randn(2, 288, 2, D, generator=g, device="cuda") for _ in range(2))
    cache = B.Cache(2, 2, D, 288, 32, 4)
    B.append(cache, k * 2.0 ** power, v, i32(0, 0))
    q = torch.zeros(2, T, 2, D, device="cuda", dtype=dtype)
    mod, lens, drafts = B.ScoreMod(softcap=cap), i32(200, 7), i32(T, T)
    mask, depth = trees(2, T, drafts, 8, chain=True)
    got = B.tree_attn(cache, q, lens, mod=mod, softmax_scale=scale)
    out, amp, reach = wide_reference(cache, q, lens, None, None, mod, scale=scale, drafts=drafts, mask=mask, depth=depth)
    check(got, out, amp, reach)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 6, 8])
@pytest.mark.parametrize("T,group", [(5, 1), (12, 1), (10, 2), (20, 2)])
@pytest.mark.parametrize("gap", [60, 99, 110, 140])
def test_blocks_far_apart_inside_a_row(gap, T, group, bits):
    """Rows whose first block is 2^gap above the others.  A cached value counts to within 2^-120 of its row's largest: the
    small blocks' outputs are right up to there, and smaller than that behind it."""
    g = torch.Generator(device="cuda").manual_seed(70 + T)
    k, v = (torch.randn(2, 304, 2, D, generator=g, device="cuda") for _ in range(2))
    high = 2.0 ** (gap // 2)
    low = high / 2.0 ** gap
    v[..., :32] *= high
    v[..., 32:] *= low
    k[..., :32] = 0.0
    k[..., 32:] *= low
    k[..., 0] = high                                    # no query looks at it
    cache = B.Cache(2, 2, D, 304, 32, bits)
    B.append(cache, k, v, i32(0, 0))
    q = torch.randn(2, T, 2 * group, D, generator=g, device="cuda").bfloat16()
    q[..., :32] = 0.0
    lens, drafts, scale = i32(280, 130), i32(T, T), 1.0 / low / math.sqrt(D)
    mask, depth = trees(2, T, drafts, 61)
    if gap > 120:                                       # the small blocks do not count: all scores are 0 then
        q.zero_()
    got = B.tree_attn(cache, q, lens, tree_mask=mask, depth=depth, softmax_scale=scale)
    out, amp, reach = wide_reference(cache, q, lens, None, None, B.ScoreMod(), scale=scale, drafts=drafts, mask=mask, depth=depth)
    check(got[..., :32] / high, out[..., :32] / high, amp[..., :32] / high, reach)
    if gap > 120:
        assert float(got[..., 32:].abs().max()) <= 2.0 ** -120 * float(v.abs().max()) + 1.01 * float(amp[..., 32:].max())
    else:
        check(got[..., 32:] / low, out[..., 32:] / low, amp[..., 32:] / low, reach)


@pytest.mark.gpu
@pytest.mark.parametrize("bits,block", ALL_FMT)
@pytest.mark.parametrize("T", [1, 5])
@pytest.mark.parametrize("top", [4.0, 0.06])
def test_fp32_queries_keep_every_bit(top, T, bits, block):
    """Queries with one channel and keys that are powers of two in it: the product is exact in three bf16 terms (two
    would lose 2^-18 of it), so the scores' error is that of three fp32 roundings; weights in three terms.  Bound: a score
    is off by 4 x 2^-24 of the largest, exp2 by 2^-22 in weight and sum, sums and third terms by 2^-22 in all."""
    g = torch.Generator(device="cuda").manual_seed(80 + T)
    n = 40
    k = torch.zeros(4, 48, 2, D, device="cuda")
    k[..., 9] = torch.tensor([1.0, -1.0, 2.0, -2.0, 0.5], device="cuda").repeat(10)[:48][None, :, None]
    v = torch.randn(4, 48, 2, D, generator=g, device="cuda")
    cache = B.Cache(4, 2, D, 48, block, bits)
    B.append(cache, k, v, i32(0, 0, 0, 0))
    q = torch.zeros(4, T, 6, D, device="cuda")
    q[..., 9] = (torch.rand(4, T, 6, generator=g, device="cuda") * 0.5 + 0.5) * (top / 2)
    lens = i32(n, 2, 3, 1)
    if T == 1:
        got = B.decode_attn_mod(cache, q[:, 0].contiguous(), lens, None, softmax_scale=1.0)[:, None]
        out, amp, _ = wide_reference(cache, q, lens, None, None, B.ScoreMod(), scale=1.0)
    else:
        drafts = i32(T, T, T, T)
        mask, depth = trees(4, T, drafts, 81, chain=True)
        got = B.tree_attn(cache, q, lens, softmax_scale=1.0)
        out, amp, _ = wide_reference(cache, q, lens, None, None, B.ScoreMod(), scale=1.0, drafts=drafts, mask=mask, depth=depth)
    bound = amp * (2 * 4 * 2.0 ** -24 * top + 2 * 2.0 ** -22 + 2.0 ** -22) + 2.0 ** -24 * out.abs() + 1e-35
    worst = float(((got.double() - out).abs() / bound).max())
    assert worst <= 1.0, f"error is {worst:.3g} of the bound"


# ----------------------------------------------------------------------------------------------- caps of any size
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("T,group", [(1, 3), (10, 1), (9, 3), (20, 3)])
@pytest.mark.parametrize("cap", [65.0, 1e5, 1e8, 1e30, 3e38])
def test_large_caps_leave_scores_alone(cap, T, group, bits, dtype):
    """The error of a capped score goes by the score, not by the cap: 2^-18 of it (the tanh's 1.5e-6 and three fp32
    roundings), on top of the product's own (24 steps of 2^-23 of the sum of |q k|, which is at least the score)."""
    cache, perm, perm_v, q, lens = long_case(7, 3, 2, group, 416, T, dtype, bits, 32, empty=0.0)
    mod, kw = B.ScoreMod(softcap=cap), dict(perm_k=perm, inv_perm_v=inverse(perm_v))
    drafts = torch.full((3,), T, dtype=torch.int32, device="cuda")
    if T == 1:
        got = B.decode_attn_mod(cache, q[:, 0].contiguous(), lens, mod, **kw)[:, None]
        out, amp, reach = wide_reference(cache, q, lens, perm, perm_v, mod)
    else:
        mask, depth = trees(3, T, drafts, 8)
        got = B.tree_attn(cache, q, lens, tree_mask=mask, depth=depth, mod=mod, **kw)
        out, amp, reach = wide_reference(cache, q, lens, perm, perm_v, mod, drafts=drafts, mask=mask, depth=depth)
    check(got, out, amp, reach * (1.0 + 2.0 ** -18 / (24 * 2.0 ** -23)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [3, 12, 40])
@pytest.mark.parametrize("grow,scale", [(2.0 ** 100, 0.0), (1.0, 1e20)])
def test_small_caps_and_large_factors(grow, scale, T, dtype):
    """The smallest cap turns every score into almost nothing, also where scale / cap or the cached magnitudes over it
    leave the fp32 range: rows of zeros (scores 0) and others weigh all they see alike."""
    g = torch.Generator(device="cuda").manual_seed(9)
    k, v = (torch.randn(2, 288, 2, D, generator=g, device="cuda") for _ in range(2))
    cache = B.Cache(2, 2, D, 288, 32, 4)
    B.append(cache, k * grow, v, i32(0, 0))
    q = torch.randn(2, T, 2, D, generator=g, device="cuda").to(dtype)
    q[:, ::2] = 0.0
    mod, lens, drafts = B.ScoreMod(softcap=1e-20), i32(200, 7), i32(T, T)
    mask, depth = trees(2, T, drafts, 8, chain=True)
    got = B.tree_attn(cache, q, lens, mod=mod, softmax_scale=scale)
    out, amp, _ = wide_reference(cache, q, lens, None, None, mod, scale=scale, drafts=drafts, mask=mask, depth=depth)
    check(got, out, amp, torch.zeros_like(amp[..., 0]))


# ----------------------------------------------------------------------------------------------- weights
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_hidden_tokens_keep_their_weights_whatever_the_query(bad, bits, dtype):
    """A query that is not finite makes its own visible tokens' weights NaN, not those of tokens it does not see."""
    cache, perm, perm_v, q, _ = long_case(10, 2, 2, 2, 480, 1, dtype, bits, 32)
    lens = i32(467, 201)
    mod = B.ScoreMod(window=77, prefix=i32(3, 9), first=i32(0, 130))
    q[0, 0, 1, 5] = bad                        # first sequence, first kv head
    mass = torch.rand(2, 2, 480, device="cuda")
    mass[0, 0, 40] = -0.0
    before = mass.clone()
    B.decode_attn_mass(cache, q[:, 0].contiguous(), lens, mass, mod=mod, perm_k=perm)
    t = torch.arange(480, device="cuda")
    for b, (n, first, prefix) in enumerate(((467, 0, 3), (201, 130, 9))):
        see = (t < prefix) | ((t >= first) & (n - 1 - t < 77) & (t < n))
        for h in range(2):
            assert torch.equal(mass[b, h, ~see].view(torch.int32), before[b, h, ~see].view(torch.int32))
            moved = mass[b, h, see]
            assert bool(torch.isnan(moved).all() if (b, h) == (0, 0) else torch.isfinite(moved).all())
    assert B.device_status() == 0


# ----------------------------------------------------------------------------------------------- the smallest calls
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits,block", ALL_FMT)
@pytest.mark.parametrize("group", [1, 8])
def test_caches_of_one_group_of_tokens(bits, block, group, dtype):
    """One head of 16 tokens, less than any tile: trees that fill it, single tokens, weights, eviction to one row."""
    g = torch.Generator(device="cuda").manual_seed(100)
    k, v = (torch.randn(1, 16, 1, D, generator=g, device="cuda") for _ in range(2))
    cache = B.Cache(1, 1, D, 16, block, bits)
    B.append(cache, k, v, i32(0))
    q = torch.randn(1, 16, group, D, generator=g, device="cuda").to(dtype)
    for n, T in ((0, 1), (0, 16), (3, 13), (15, 1), (7, 2)):
        qt, drafts = q[:, :T].contiguous(), i32(T)
        mask, depth = trees(1, T, drafts, 101)
        got = B.tree_attn(cache, qt, i32(n), tree_mask=mask, depth=depth)
        check(got, *wide_reference(cache, qt, i32(n), None, None, B.ScoreMod(), drafts=drafts, mask=mask, depth=depth))
    for n in (1, 16):
        q1, mass, w = q[:, 0].contiguous(), torch.zeros(1, 1, 16, device="cuda"), torch.zeros(1, 1, 16, dtype=torch.float64, device="cuda")
        got = B.decode_attn_mass(cache, q1, i32(n), mass)
        check(got[:, None], *wide_reference(cache, q[:, :1], i32(n), None, None, B.ScoreMod(), weights=w))
        assert float((mass - w).abs().max()) <= 1e-5 * group
    keep = int(mass[0, 0].argmax())
    kept, new = B.evict(cache, i32(16), mass, 1)
    assert kept.tolist() == [[[keep]]] and new.tolist() == [1]
    assert B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 6, 8])
def test_trees_far_into_a_long_cache(bits):
    """Offsets past 32 bits in every width of tree and with weights: the second head's rows lie 3 GB and more into a plane,
    its last ones more than twice that."""
    H, S = 2, (1 << 25) + (1 << 24)
    n = S - 80
    g = torch.Generator(device="cuda").manual_seed(110)
    k, v = (torch.randn(1, 304, H, D, generator=g, device="cuda") for _ in range(2))
    small, cache = B.Cache(1, H, D, 304, 32, bits), B.Cache(1, H, D, S, 32, bits)
    B.append(small, k, v, i32(0))
    index = torch.arange(304, dtype=torch.int32, device="cuda")[None].contiguous()
    B.gather_rows(small, index, i32(304), dst=cache, dst_base=i32(n - 264))
    assert H * S * cache.fmt.row_m > 1 << 32
    mod = B.ScoreMod(window=250)
    for T, group, dtype in ((3, 2, torch.bfloat16), (12, 1, torch.bfloat16), (10, 3, torch.bfloat16), (20, 3, torch.bfloat16),
                            (5, 2, torch.float32)):
        q, drafts = torch.randn(1, T, H * group, D, generator=g, device="cuda").to(dtype), i32(T)
        mask, depth = trees(1, T, drafts, 111)
        got = B.tree_attn(cache, q, i32(n), tree_mask=mask, depth=depth, mod=mod)
        want = B.tree_attn(small, q, i32(264), tree_mask=mask, depth=depth, mod=mod)
        ref = wide_reference(small, q, i32(264), None, None, mod, drafts=drafts, mask=mask, depth=depth)
        check(got, *ref)
        check(want, *ref)
    q1 = q[:, 0].contiguous()
    mass, few = torch.zeros(1, H, S, device="cuda"), torch.zeros(1, H, 304, device="cuda")
    B.decode_attn_mass(cache, q1, i32(n), mass, mod=mod)
    B.decode_attn_mass(small, q1, i32(264), few, mod=mod)
    assert float((mass[:, :, n - 264:n + 40] - few).abs().max()) <= 1e-6 * 2
    assert float(mass[:, :, :n - 264].abs().max()) == 0.0 and B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 6, 8])
@pytest.mark.parametrize("T,group", [(1, 1), (3, 2), (12, 1), (10, 3), (20, 3)])
def test_orders_that_are_no_permutation_stay_inside_the_output(T, group, bits):
    """Channel orders that name a channel twice, or none that exists: the results are unspecified, the memory around them is
    left alone."""
    cache, _, _, q, lens = long_case(120, 4, 3, group, 416, T, torch.bfloat16, bits, 32)
    around = torch.full((3, *q.shape), 7.0, dtype=q.dtype, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(121)
    for order in (torch.zeros(3, D), torch.full((3, D), -1), torch.full((3, D), 1 << 30),
                  torch.randint(-2 ** 31, 2 ** 31 - 1, (3, D), generator=g, device="cuda")):
        order = order.to(torch.int32).cuda()
        around.fill_(7.0)
        B.tree_attn(cache, q, lens, perm_k=order, inv_perm_v=order, out=around[1])
        assert bool((around[0] == 7.0).all()) and bool((around[2] == 7.0).all())
    assert B.device_status() == 0


def test_channel_table_entries_are_cut_to_a_channel():
    with open(os.path.join(build.CSRC, "attn_umma.cuh")) as f:
        assert "chan[slot_of] & (D - 1)" in f.read()


# ----------------------------------------------------------------------------------------------- refusals
def test_queries_of_another_rank_are_refused():
    """One token's queries given as a tree's would be read far past their end, a tree's as one token's in part."""
    cache = B.Cache(2, 2, D, 64, 32, 4, device="cpu")
    lens, mass = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 2, 64)
    one, tree = torch.zeros(2, 4, D), torch.zeros(2, 3, 4, D)
    for q in (one, tree[:, 0, 0], tree[None]):
        with pytest.raises(ValueError, match="expected .B, T, H_q, d."):
            B.tree_attn(cache, q, lens)
    for q in (tree, one[:, 0]):
        with pytest.raises(ValueError, match="expected .B, H_q, d."):
            B.decode_attn_mod(cache, q, lens, None)
        with pytest.raises(ValueError, match="expected .B, H_q, d."):
            B.decode_attn_mass(cache, q, lens, mass)


@pytest.mark.gpu
def test_queries_of_another_rank_launch_nothing():
    cache, perm, _, q, lens = long_case(6, 2, 2, 2, 64, 4, torch.bfloat16, 4, 32)
    mass, before = torch.zeros(2, 2, 64, device="cuda"), B.launch_count()
    for call in (lambda: B.tree_attn(cache, q[:, 0].contiguous(), lens), lambda: B.decode_attn_mod(cache, q, lens, None),
                 lambda: B.decode_attn_mass(cache, q, lens, mass)):
        with pytest.raises(ValueError, match="expected"):
            call()
    assert B.launch_count() == before


def test_caches_that_share_memory_across_planes_are_refused():
    """Another cache whose K lies where the source's V does would be written while it is read."""
    L, vp = B.lib(), C.c_void_p
    f, small = B.Format(1, 2, 128, 64, 32, 4), B.Format(1, 2, 128, 32, 32, 4)
    src = B.CacheStruct(f, 0x100000, 0x200000, 0x300000, 0x400000)          # 8192, 512, 8192, 512 bytes
    good = [0x500000, 0x600000, 0x700000, 0x800000]
    before = B.launch_count()
    for i in range(4):
        for at in (0x100000, 0x200000, 0x300000, 0x400000, 0x101ff0, 0x2001f0, 0x301ff0, 0x4001f0, 0x300000 - 16):
            planes = good[:i] + [at] + good[i + 1:]
            dst = B.CacheStruct(small, *planes)
            assert L.kvbfp_gather_rows(C.byref(src), C.byref(dst), vp(16), 1, 4, vp(16), None, None, None) == B.ERR_INVALID_ARG
            assert L.kvbfp_evict(C.byref(src), vp(16), vp(0x10000), 16, 4, 4, C.byref(dst), vp(0x20000), vp(16), vp(16), None) == B.ERR_INVALID_ARG
    assert B.launch_count() == before


def test_index_lists_past_two_to_the_thirty_are_refused():
    """The kernel counts rows of a list in 32 bits, 128 at a time."""
    L, vp = B.lib(), C.c_void_p
    src = B.CacheStruct(B.Format(1, 2, 128, 64, 32, 4), 0x100000, 0x200000, 0x300000, 0x400000)
    for n in ((1 << 30) + 1, (1 << 31) - 1):
        assert L.kvbfp_gather_rows(C.byref(src), C.byref(src), vp(16), 1, n, vp(16), None, None, None) == B.ERR_UNSUPPORTED


def test_evict_takes_both_destinations_or_none():
    """Weights of their own without a cache of their own were left empty, and the given ones overwritten, without a word."""
    cache, small = (B.Cache(1, 2, D, n, 32, 4, device="cpu") for n in (64, 32))
    lens, mass, other = torch.zeros(1, dtype=torch.int32), torch.zeros(1, 2, 64), torch.zeros(1, 2, 32)
    with pytest.raises(ValueError, match="dst_mass"):
        B.evict(cache, lens, mass, 16, dst_mass=other)
    with pytest.raises(ValueError, match="dst_mass"):
        B.evict(cache, lens, mass, 16, dst=small)
