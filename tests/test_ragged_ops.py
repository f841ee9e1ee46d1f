"""Attention of ragged batches over contiguous and paged caches (causal, window, first tokens), the norm / rotation / cache
write in one step, and the bookkeeping of pages, against plain forms in 64 bits (numpy models for the pages)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2403_20137_b200 import binding as B

D = 128
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step, relative
FMT = [(4, 16), (4, 32), (4, 128), (6, 32), (6, 64), (8, 16), (8, 32)]


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def inverse(perm):
    inv = torch.empty_like(perm)
    inv.scatter_(1, perm.long(), torch.arange(D, dtype=torch.int32, device=perm.device).expand_as(perm))
    return inv


def perms(heads, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.stack([torch.randperm(D, generator=g) for _ in range(heads)]).to(torch.int32).cuda() for _ in range(2)]


def fill(cache, seed, perm=None, perm_v=None, scale=1.0):
    """Seeded rows everywhere in a cache (or pool), a few key channels loud."""
    f = cache.fmt
    g = torch.Generator().manual_seed(seed)
    k = torch.randn(f.batch, f.max_seq, f.n_kv_heads, D, generator=g) * scale
    v = torch.randn(f.batch, f.max_seq, f.n_kv_heads, D, generator=g) * scale
    k[..., [3, 77, 120]] *= 4.0
    B.append(cache, k.cuda(), v.cuda(), torch.zeros(f.batch, dtype=torch.int32, device="cuda"), perm_k=perm, perm_v=perm_v)


def paged(lens, heads, page, bits, block, seed, perm=None, perm_v=None, extra=3, scale=1.0, cols=None):
    """A pool whose pages lie in random order, the sequences' tables (other entries -1)."""
    rng = np.random.default_rng(seed)
    need = [(n + page - 1) // page for n in lens]
    n_pages = sum(need) + extra
    order = rng.permutation(n_pages)
    table = np.full((len(lens), cols or max(max(need), 1)), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    cache = B.Cache(n_pages, heads, D, page, block, bits)
    fill(cache, seed, perm, perm_v, scale)
    refs = np.zeros(n_pages, np.int32)
    refs[order[:at]] = 1
    pool = B.PagePool.of(torch.from_numpy(table).cuda(), torch.from_numpy(refs).cuda(), i32(*lens), n_pages, page)
    return cache, pool


def rows_of(cache, pool, which, b, n, perm):
    """The first n rows of sequence b in channel order, fp64 [n, H, D]."""
    x = B.dequant_all(cache, which, cache.fmt.max_seq, perm=perm).double()
    if pool is None:
        return x[b, :n]
    t = torch.arange(n, device="cuda")
    return x[pool.table[b, t // pool.page_tokens].long().clamp_min(0), t % pool.page_tokens]


def reference(cache, pool, q, news, lens, perm, perm_v, window=0, sink=0, scale=0.0):
    """-> out, the sum of p|v| per output, the largest sum of |q k| scale per row; fp64, [n, Hq, D]."""
    H = cache.fmt.n_kv_heads
    Hq = q.shape[1]
    G = Hq // H
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    amp, reach = torch.zeros_like(out), torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    scale = scale or 1.0 / math.sqrt(D)
    row = 0
    for b, (new, n) in enumerate(zip(news, lens)):
        k, v = (rows_of(cache, pool, w, b, n, p) for w, p in (("k", perm), ("v", perm_v)))
        pos = torch.arange(n - new, n, device="cuda")[:, None]
        t = torch.arange(n, device="cuda")
        see = t <= pos
        if window:
            see &= (pos - t < window) | (t < sink)
        some = see.any(-1)
        for hq in range(Hq):
            x = q[row:row + new, hq].double()
            s = (x @ k[:, hq // G].T) * scale
            p = torch.softmax(s.masked_fill(~see, -math.inf), -1)
            p = torch.where(some[:, None], p, 0.0)
            out[row:row + new, hq] = p @ v[:, hq // G]
            amp[row:row + new, hq] = p @ v[:, hq // G].abs()
            if n:
                reach[row:row + new, hq] = ((x.abs() @ k[:, hq // G].abs().T) * scale).masked_fill(~see, 0.0).amax(-1)
        row += new
    return out, amp, reach


def check(got, out, amp, reach):
    """Error bound per output.  Scores: fp32 products in chains of up to 24 tensor-core steps that cut (2^-23 of the running sum
    of |q k| each; fp32 queries drop 2^-25 of q); a score error d changes a weight by d relative, an output by 2 d sum(p|v|).
    Weights are rounded to bf16 (half a step) or, for fp32 queries, cut to three bf16 terms (2^-16 allows for two), exp2 and the
    sums add 2^-20; the output is rounded once."""
    d = 24 * 2.0 ** -23 * reach
    w = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -16
    bound = amp * (2 * d[..., None] + w + 2.0 ** -20) * 1.01 + HALF[got.dtype] * out.abs() * 1.01 + 1e-35
    worst = float(((got.double() - out).abs() / bound).max())
    assert bool(torch.isfinite(got).all()) and worst <= 1.0, f"error is {worst:.3g} of the bound"


def batch_of(news, lens, heads, group, bits, block, page, dtype, seed, scale=1.0):
    """(cache, pool, q, starts, lens tensor, permutations)"""
    perm, perm_v = perms(heads, seed)
    if page:
        cache, pool = paged(lens, heads, page, bits, block, seed, perm, perm_v, scale=scale)
    else:
        cache, pool = B.Cache(len(lens), heads, D, max(16, (max(lens) + 15) // 16 * 16), block, bits), None
        fill(cache, seed, perm, perm_v, scale)
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn(sum(news), heads * group, D, generator=g).to(dtype).cuda()
    starts = i32(*np.concatenate([[0], np.cumsum(news)]).tolist())
    return cache, pool, q, starts, i32(*lens), perm, perm_v


def attend(args, news, **kw):
    cache, pool, q, starts, lens, perm, perm_v = args
    return B.ragged_attn(cache, q, starts, lens, max(news), perm_k=perm, inv_perm_v=inverse(perm_v), pool=pool, **kw)


def attend_and_check(args, news, lens, window=0, sink=0, scale=0.0):
    got = attend(args, news, window=window, n_sink=sink, softmax_scale=scale)
    check(got, *reference(args[0], args[1], args[2], news, lens, args[5], args[6], window, sink, scale))
    assert B.device_status() == 0
    return got


# ----------------------------------------------------------------------------------------------- attention
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits,block", FMT)
@pytest.mark.parametrize("page,group", [(0, 1), (16, 4), (64, 3), (256, 8)])
def test_ragged_attn_formats(bits, block, page, group, dtype):
    """Single tokens, short and long chunks and whole prompts in one batch, in every format and page size."""
    news, lens = [1, 3, 40, 150, 1], [300, 3, 129, 150, 1]
    args = batch_of(news, lens, 2, group, bits, block, page, dtype, bits * 7 + block + page)
    attend_and_check(args, news, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page", [0, 16, 32, 128])
@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (17, 4), (64, 64), (100, 300), (5000, 9), (130, 17)])
def test_ragged_attn_windows(window, sink, page, dtype):
    """Windows shorter and longer than a tile, first tokens that end inside one, overlap the window or cover everything."""
    news, lens = [1, 1, 8, 200, 33, 1], [700, 20, 500, 400, 33, 129]
    args = batch_of(news, lens, 1, 2, 4, 32, page, dtype, window + sink)
    attend_and_check(args, news, lens, window, sink, scale=0.11)


@pytest.mark.gpu
@pytest.mark.parametrize("news,lens", [([1], [1]), ([0, 1, 0], [5, 2, 0]), ([2, 0, 7], [2, 0, 7]), ([1] * 70, [13 * (b % 9) + 1 for b in range(70)]),
                                       ([5, 300, 1, 0, 64], [64, 300, 65, 9, 1000])])
@pytest.mark.parametrize("dtype,page", [(torch.bfloat16, 16), (torch.float32, 64), (torch.bfloat16, 0)])
def test_ragged_attn_batches(news, lens, dtype, page):
    """One token, sequences without new tokens, empty sequences, many sequences."""
    args = batch_of(news, lens, 2, 2, 4, 32, page, dtype, len(news))
    attend_and_check(args, news, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 6, 8])
@pytest.mark.parametrize("group,new", [(1, 1), (1, 128), (1, 129), (2, 127), (4, 65), (5, 51), (8, 33), (3, 300)])
def test_ragged_attn_row_counts(group, new, bits):
    """Row counts around the sizes that kernels tile by."""
    news, lens = [new, 1], [new + 190, 257]
    args = batch_of(news, lens, 2, group, bits, 32, 32, torch.bfloat16, new + group)
    attend_and_check(args, news, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 6, 8])
@pytest.mark.parametrize("group,news", [(1, [8, 9, 16, 17, 4, 5]), (4, [2, 3, 4, 5, 1, 0]), (8, [1, 2, 3, 1, 2, 3]), (5, [3, 4, 1, 2, 0, 3]), (4, [4])])
def test_ragged_attn_rows_around_the_borders(group, news, bits):
    """Rows per kv head around the numbers that choose a kernel and its items, every way of hinting at them."""
    lens = [n + 170 + 61 * b for b, n in enumerate(news)]
    args = batch_of(news, lens, 2, group, bits, 32, 32, torch.bfloat16, group + bits)
    cache, pool, q, starts, n, perm, perm_v = args
    ref = reference(cache, pool, q, news, lens, perm, perm_v)
    for hint in (0, 1, 2, 3, max(news), 16, 17, 1000):
        check(B.ragged_attn(cache, q, starts, n, hint, perm_k=perm, inv_perm_v=inverse(perm_v), pool=pool), *ref)
    assert B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("hint", [0, 1, 8])
@pytest.mark.parametrize("bits,block", FMT)
@pytest.mark.parametrize("group,news", [(1, [1, 4, 3]), (3, [1, 2, 1]), (4, [1, 1, 2]), (8, [1, 1, 1]), (5, [1, 0, 1])])
def test_ragged_attn_weights_of_few_rows(group, news, bits, block, hint):
    """Up to eight bf16 rows per kv head keep 16 bits of the weights.  Terms as in check(): two bf16 terms leave half a step of half a
    step, 2^-16; a small scale, so that the bound of the scores does not hide it (weights all near one: outputs that cancel)."""
    lens = [100, 77, 130]
    args = batch_of(news, lens, 2, group, bits, block, 32, torch.bfloat16, group + bits + block)
    cache, pool, q, starts, n, perm, perm_v = args
    got = B.ragged_attn(cache, q, starts, n, hint, perm_k=perm, inv_perm_v=inverse(perm_v), pool=pool, softmax_scale=0.002).double()
    out, amp, reach = reference(cache, pool, q, news, lens, perm, perm_v, scale=0.002)
    bound = amp * (2 * 24 * 2.0 ** -23 * reach[..., None] + 2.0 ** -16 + 2.0 ** -20) * 1.01 + 2.0 ** -8 * out.abs() * 1.01
    worst = float(((got - out).abs() / bound).max())
    assert worst <= 1.0, f"error is {worst:.3g} of the bound"
    assert B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ragged_attn_long(dtype):
    """Work for every worker, entries that span several of them, ragged."""
    news, lens = [1, 700 if dtype == torch.bfloat16 else 20, 1, 9], [9000, 4100, 33, 6000]
    args = batch_of(news, lens, 4, 2, 4, 32, 64, dtype, 3)
    attend_and_check(args, news, lens)
    attend_and_check(args, news, lens, window=1500, sink=4)


@pytest.mark.gpu
def test_ragged_attn_equals_token_by_token():
    """A chunk gives what its tokens give one after the other: each row within the bound of the same reference."""
    news, lens = [40], [333]
    args = batch_of(news, lens, 2, 4, 8, 32, 32, torch.bfloat16, 8)
    cache, pool, q, starts, _, perm, perm_v = args
    ref = reference(cache, pool, q, news, lens, perm, perm_v, 100, 5)
    for i in range(0, 40, 7):
        one = B.ragged_attn(cache, q[i:i + 1].contiguous(), i32(0, 1), i32(333 - 40 + i + 1), 1, window=100, n_sink=5, perm_k=perm,
                            inv_perm_v=inverse(perm_v), pool=pool)
        check(one, *(x[i:i + 1] for x in ref))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ragged_attn_max_new_is_only_a_hint(dtype):
    news, lens = [1, 90, 7], [200, 300, 7]
    args = batch_of(news, lens, 2, 2, 4, 32, 32, dtype, 9)
    cache, pool, q, starts, n, perm, perm_v = args
    ref = reference(cache, pool, q, news, lens, perm, perm_v)
    for hint in (0, 1, 90, 100000):
        check(B.ragged_attn(cache, q, starts, n, hint, perm_k=perm, inv_perm_v=inverse(perm_v), pool=pool), *ref)


@pytest.mark.gpu
@pytest.mark.parametrize("new", [1, 200])
def test_ragged_attn_leaves_other_rows(new):
    """Rows of q behind the last sequence are neither read nor written; freed pages outside the window are not needed."""
    news, lens = [new, 2], [900, 50]
    cache, pool, q, starts, n, perm, perm_v = batch_of(news, lens, 2, 2, 4, 32, 32, torch.bfloat16, 4)
    ref = reference(cache, pool, q, news, lens, perm, perm_v, 100, 40)
    more = torch.full((q.shape[0] + 5, 4, D), math.nan, dtype=torch.bfloat16, device="cuda")
    more[:q.shape[0]] = q
    out = torch.full_like(more, 7.0)
    B.pages_free(pool, lo=i32(40, 40), hi=i32(900 - new - 99, 0))
    assert int((pool.table[0] < 0).sum()) >= 10
    B.ragged_attn(cache, more, starts, n, new, window=100, n_sink=40, perm_k=perm, inv_perm_v=inverse(perm_v), pool=pool, out=out)
    assert bool((out[q.shape[0]:] == 7.0).all())
    check(out[:q.shape[0]], *ref)
    assert B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page", [0, 16])
def test_ragged_attn_flags(page, dtype):
    """Lengths beyond the cache, more new tokens than cached ones, a missing page: flagged; the other sequences are right."""
    news, lens = [3, 60, 2], [100, 60, 80]
    args = batch_of(news, lens, 1, 2, 4, 32, page, dtype, 5)
    cache, pool, q, starts, n, perm, perm_v = args
    ref = reference(cache, pool, q, news, lens, perm, perm_v)
    kw = dict(perm_k=perm, inv_perm_v=inverse(perm_v), pool=pool)
    n2 = n.clone()
    n2[1] = 20                                  # 40 of its tokens would stand before the first position
    got = B.ragged_attn(cache, q, starts, n2, 60, out=torch.full_like(q, 5.0), **kw)
    assert bool((got[3:43] == 0).all())
    short = reference(cache, pool, q[43:63].contiguous(), [0, 20, 0], [0, 20, 0], perm, perm_v)
    check(got[43:63], *short)
    check(got[:3], *(x[:3] for x in ref))
    check(got[63:], *(x[63:] for x in ref))
    assert B.device_status() == 0
    n2[1] = 10 ** 9
    got = B.ragged_attn(cache, q, starts, n2, 60, **kw)
    check(got[:3], *(x[:3] for x in ref))
    check(got[63:], *(x[63:] for x in ref))
    assert B.device_status() == B.FLAG_POSITION
    if pool is not None:
        for bad in (-1, 10 ** 6):
            pool.table[1, 1] = bad
            got = B.ragged_attn(cache, q, starts, n, 60, **kw)
            check(got[:3], *(x[:3] for x in ref))
            check(got[63:], *(x[63:] for x in ref))
            assert B.device_status() == B.FLAG_POSITION


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ragged_attn_starts_that_decrease(dtype):
    """Flagged, nothing is attended; the next call is served."""
    news, lens = [3, 60, 2], [100, 60, 80]
    args = batch_of(news, lens, 1, 2, 4, 32, 16, dtype, 5)
    cache, pool, q, starts, n, perm, perm_v = args
    n = i32(100, 66, 80)                     # (no tokens before the first position)
    for bad in (i32(0, 63, 3, 65), i32(5, 0, 65, 65), i32(0, 3, 63, 62)):
        for hint in (2, 60):
            got = B.ragged_attn(cache, q, bad, n, hint, perm_k=perm, inv_perm_v=inverse(perm_v), pool=pool, out=torch.full_like(q, 5.0))
            assert bool((got == 5.0).all())
            assert B.device_status() == B.FLAG_POSITION
    attend_and_check(args, news, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hint", [1, 20000])
def test_ragged_attn_many_rows_before_the_first_position(dtype, hint):
    """Long sequences whose lengths were not raised, among others: their rows are zeros (all but the last seven of the third),
    the others' right.  More than 32 sequences."""
    news, lens = [1, 20000, 3000, 5] + [0, 2] * 20, [700, 0, 7, 90] + [0, 0] * 20
    some = [1, 0, 7, 5] + [0] * 40
    g = torch.Generator().manual_seed(3)
    args = batch_of(some, lens, 1, 4, 4, 32, 16, dtype, 3)
    cache, pool, few, _, n, perm, perm_v = args
    ref = reference(cache, pool, few, some, lens, perm, perm_v)
    q = torch.randn(sum(news), 4, D, generator=g).to(dtype).cuda()
    at = torch.cat([torch.arange(1), torch.arange(22994, 23001), torch.arange(23001, 23006)]).cuda()
    q[at] = few
    starts = i32(*np.concatenate([[0], np.cumsum(news)]).tolist())
    out = torch.full((q.shape[0] + 3, 4, D), 5.0, dtype=dtype, device="cuda")
    got = B.ragged_attn(cache, torch.cat([q, q[:3]]), starts, n, hint, perm_k=perm, inv_perm_v=inverse(perm_v), pool=pool, out=out)
    check(got[at], *ref)
    rest = torch.ones(got.shape[0], dtype=torch.bool, device="cuda")
    rest[at], rest[-3:] = False, False
    assert bool((got[rest] == 0).all()) and bool((got[-3:] == 5.0).all())
    assert B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ragged_attn_largest_window(dtype):
    """Windows and numbers of first tokens up to the largest integer, rows before the first position among them."""
    news, lens = [40, 1], [90, 70]
    cache, pool, q, starts, n, perm, perm_v = batch_of(news, lens, 1, 2, 4, 32, 16, dtype, 5)
    n[0] = 30                                            # ten tokens before the first position
    ref = reference(cache, pool, q[10:].contiguous(), [30, 1], [30, 70], perm, perm_v)
    for window, sink in ((2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (96, 3), (1, 2 ** 31 - 1), (95, 0)):
        got = B.ragged_attn(cache, q, starts, n, 40, window=window, n_sink=sink, perm_k=perm, inv_perm_v=inverse(perm_v), pool=pool)
        assert bool((got[:10] == 0).all())
        check(got[10:], *ref)
    assert B.device_status() == 0


@pytest.mark.gpu
def test_ragged_attn_long_prompts_are_not_refused():
    """131072 new tokens of 32 heads count few enough items: a batch of that size whose sequences are empty."""
    cache = B.Cache(1, 8, D, 131072, 32, 4)
    q = torch.empty(131072, 32, D, dtype=torch.bfloat16, device="cuda")
    out = torch.full((131072, 32, D), 3.0, dtype=torch.bfloat16, device="cuda")
    for hint in (131072, 0):
        B.ragged_attn(cache, q, i32(0, 0), i32(0), hint, out=out)
    assert bool((out == 3.0).all()) and B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits,block", [(4, 16), (4, 32), (6, 64), (8, 32)])
@pytest.mark.parametrize("page", [0, 16, 128])
def test_ragged_attn_hidden_rows_may_hold_anything(page, bits, block, dtype):
    """Rows behind the sequences, in pages of no sequence, before the window: all ones, exponent bytes too (no row that was
    written holds them)."""
    news, lens, window, sink = [1, 130, 5], [201, 390, 77], 64, 5
    cache, pool, q, starts, n, perm, perm_v = batch_of(news, lens, 2, 2, bits, block, page, dtype, 31)
    ref = reference(cache, pool, q, news, lens, perm, perm_v, window, sink)
    seen = torch.zeros(cache.fmt.batch, cache.fmt.max_seq, dtype=torch.bool, device="cuda")
    for b, (new, ln) in enumerate(zip(news, lens)):
        for t in [*range(sink), *range(max(ln - new - window + 1, 0), ln)]:
            if pool is None:
                seen[b, t] = True
            else:
                seen[int(pool.table[b, t // page]), t % page] = True
    for name in ("k_mant", "k_exp", "v_mant", "v_exp"):
        x = getattr(cache, name)
        x.masked_fill_(~seen[:, None, :, None], 255)
    kw = dict(perm_k=perm, inv_perm_v=inverse(perm_v), pool=pool)
    check(B.ragged_attn(cache, q, starts, n, 130, window=window, n_sink=sink, **kw), *ref)
    check(B.ragged_attn(cache, q, starts, n, 1, window=window, n_sink=sink, **kw), *ref)
    assert B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ragged_attn_bad_queries_stay_alone(dtype):
    """A query of NaN or infinities spoils its own row only."""
    news, lens = [1, 200, 2], [90, 333, 70]
    args = batch_of(news, lens, 2, 2, 4, 32, 32, dtype, 32)
    q = args[2]
    ref = reference(args[0], args[1], q, news, lens, args[5], args[6])
    good = torch.ones(q.shape[:2], dtype=torch.bool, device="cuda")
    for at, value in (((0, 1), math.nan), ((50, 2), math.inf), ((51, 0), -math.inf), ((201, 3), math.nan)):
        q[at[0], at[1], 17:40] = value
        good[at] = False
    got = attend(args, news)
    check(got[good], *(x[good] for x in ref))
    assert not bool(torch.isfinite(got[~good]).all(-1).any())


@pytest.mark.gpu
def test_ragged_attn_graphs_share_a_workspace():
    """Two captured calls of different batches over one workspace, replayed in turn."""
    calls = []
    for news, lens, seed in (([1, 300, 2], [700, 300, 90], 41), ([9, 1, 64], [9, 5000, 600], 42)):
        args = batch_of(news, lens, 2, 2, 4, 32, 32, torch.bfloat16, seed)
        calls.append((args, news, reference(args[0], args[1], args[2], news, lens, args[5], args[6])))
    need = max(B.ragged_workspace_bytes(a[0].fmt, 3, 4, sum(n)) for a, n, _ in calls)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(a[2]) for a, _, _ in calls]
    kws = [dict(out=o, workspace=ws) for o in outs]
    for (a, n, _), kw in zip(calls, kws):
        attend(a, n, **kw)
    torch.cuda.synchronize()
    graphs = []
    for (a, n, _), kw in zip(calls, kws):
        inv = inverse(a[6])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.ragged_attn(a[0], a[2], a[3], a[4], max(n), perm_k=a[5], inv_perm_v=inv, pool=a[1], **kw)
        graphs.append((g, inv))
    for i in (0, 1, 1, 0, 1, 0):
        outs[i].zero_()
        graphs[i][0].replay()
        check(outs[i], *calls[i][2])
    assert B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [2.0 ** 90, 2.0 ** -90])
def test_ragged_attn_large_and_small_values(scale):
    news, lens = [1, 100], [150, 130]
    cache, pool, q, starts, n, perm, perm_v = batch_of(news, lens, 1, 2, 4, 32, 16, torch.float32, 6, scale=scale)
    q = q / scale
    for dt in (torch.float32, torch.bfloat16):
        x = q.to(dt)
        got = B.ragged_attn(cache, x, starts, n, 100, perm_k=perm, inv_perm_v=inverse(perm_v), pool=pool)
        out, amp, reach = reference(cache, pool, x, news, lens, perm, perm_v)
        check(got / scale, out / scale, amp / scale, reach)


@pytest.mark.gpu
def test_ragged_attn_large_scores():
    """Scores of some thousands: one token takes the weight, nothing overflows."""
    news, lens = [1, 150], [300, 400]
    args = batch_of(news, lens, 1, 4, 4, 32, 32, torch.bfloat16, 61)
    attend_and_check(args, news, lens, scale=20.0)


@pytest.mark.gpu
def test_ragged_attn_offsets_past_32_bits():
    """A pool whose planes pass 2^32 bytes: pages at its end."""
    heads, page = 8, 1024
    n_pages = (1 << 32) // (heads * page * 64) + 8
    cache = B.Cache(n_pages, heads, D, page, 32, 4, fill=0)
    small = B.Cache(4, heads, D, page, 32, 4)
    fill(small, 1)
    for name in ("k_mant", "k_exp", "v_mant", "v_exp"):
        getattr(cache, name)[-4:] = getattr(small, name)
    table = i32(n_pages - 1, n_pages - 3, n_pages - 2, n_pages - 4).reshape(2, 2)
    pool = B.PagePool.of(table, None, i32(2000, 1500), n_pages, page)
    spool = B.PagePool.of(i32(3, 1, 2, 0).reshape(2, 2), None, i32(2000, 1500), 4, page)
    q = torch.randn(301, 8, D, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    args = dict(starts=i32(0, 1, 301), seq_lens=i32(2000, 1500), max_new=300)
    a = B.ragged_attn(cache, q, pool=pool, **args)
    assert torch.equal(a, B.ragged_attn(small, q, pool=spool, **args))
    # and a write there
    for c, p in ((cache, pool), (small, spool)):
        B.norm_rope_append(c, None, q, q, args["starts"], args["seq_lens"], pool=p)
    for name in ("k_mant", "k_exp", "v_mant", "v_exp"):
        assert torch.equal(getattr(cache, name)[-4:], getattr(small, name))
    # and a copy from and to the end
    B.pages_copy(cache, i32(n_pages - 1, 0, 1, n_pages - 4).reshape(2, 2))
    assert torch.equal(cache.k_mant[0], small.k_mant[3]) and torch.equal(cache.v_exp[0], small.v_exp[3])
    assert bool((cache.v_mant[-4] == 0).all())
    assert B.device_status() == 0


# ----------------------------------------------------------------------------------------------- write
def rotated64(x, w, eps, theta, half, pos):
    """Norm (w None: none) and rotation (theta None: none) of rows [n, H, D] in 64 bits."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    if theta is None:
        return x
    ang = pos.double()[:, None] * theta
    cs, sn = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
    a, b = (x[..., :64], x[..., 64:]) if half else (x[..., 0::2], x[..., 1::2])
    y = torch.empty_like(x)
    if half:
        y[..., :64], y[..., 64:] = a * cs - b * sn, a * sn + b * cs
    else:
        y[..., 0::2], y[..., 1::2] = a * cs - b * sn, a * sn + b * cs
    return y


def cast64(y, bits, block):
    """Mantissas and exponent bytes of rows in slot order [..., D]."""
    m, e = y.cpu().numpy().reshape(*y.shape[:-1], D // block, block), None
    amax = np.abs(m).max(-1)
    e = np.where(amax > 0, np.frexp(amax)[1] - 1, -127).clip(-127, 127)
    top = (1 << (bits - 1)) - 1
    q = np.rint(np.ldexp(m, (-(e - (bits - 2)))[..., None])).clip(-top, top).astype(np.int64)
    return q.reshape(y.shape), (e + 127).astype(np.uint8)


def fields(mant, bits):
    """Mantissas of packed rows, field by field from the bit stream."""
    raw = mant.cpu().numpy().astype(np.int64)
    raw = np.concatenate([raw, np.zeros_like(raw[..., :1])], -1)
    bit = np.arange(D) * bits
    return (((raw[..., bit // 8] | (raw[..., bit // 8 + 1] << 8)) >> (bit % 8)) & ((1 << bits) - 1)) - (1 << (bits - 1))


def write_case(news, lens, hq, heads, bits, block, page, dtype, seed, packed=True):
    rng = torch.Generator().manual_seed(seed)
    perm, perm_v = perms(heads, seed)
    n = sum(news)
    x = torch.randn(n, hq + 2 * heads, D, generator=rng)
    x[:, hq:hq + heads, [3, 77, 120]] *= 4.0
    x = x.to(dtype).cuda()
    if page:
        cache, pool = paged(lens, heads, page, bits, block, seed)
    else:
        cache, pool = B.Cache(len(lens), heads, D, max(16, (max(lens) + 15) // 16 * 16), block, bits), None
        fill(cache, seed)
    q, k, v = x[:, :hq], x[:, hq:hq + heads], x[:, hq + heads:]
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    w = [1.0 + 0.3 * torch.randn(D, generator=rng).cuda() for _ in range(2)]
    theta = 10000.0 ** (-2.0 * torch.arange(64, dtype=torch.float64, device="cuda") / D)
    starts = i32(*np.concatenate([[0], np.cumsum(news)]).tolist())
    pos = torch.cat([torch.arange(n - m, n) for n, m in zip(lens, news)]).cuda()
    return cache, pool, q, k, v, w, theta, starts, i32(*lens), pos, perm, perm_v


def planes(cache):
    return [getattr(cache, n).clone() for n in ("k_mant", "k_exp", "v_mant", "v_exp")]


def check_write(cache, pool, before, k64, v64, news, lens, perm, perm_v, bits, block):
    """The new tokens' codes are those of the formula, every other byte is as before."""
    heads = cache.fmt.n_kv_heads
    row, n = 0, 0
    at = []
    for b, (new, ln) in enumerate(zip(news, lens)):
        for i in range(new):
            p = ln - new + i
            at.append((int(pool.table[b, p // pool.page_tokens]), p % pool.page_tokens) if pool is not None else (b, p))
    pg = torch.tensor([x[0] for x in at], device="cuda")
    rw = torch.tensor([x[1] for x in at], device="cuda")
    for x64, pm, mant, exp8, old in ((k64, perm, cache.k_mant, cache.k_exp, before[:2]), (v64, perm_v, cache.v_mant, cache.v_exp, before[2:])):
        slots = x64 if pm is None else x64.gather(-1, pm.long()[None].expand(x64.shape[0], heads, D))
        m, e = cast64(slots, bits, block)
        assert np.array_equal(exp8[pg, :, rw].cpu().numpy(), e)
        assert np.array_equal(fields(mant[pg, :, rw], bits), m)
        for now, was in ((mant, old[0]), (exp8, old[1])):
            was[pg, :, rw] = now[pg, :, rw]
            assert torch.equal(now, was)


def check_q(got, want):
    """fp32: the bound of kernels' own error, 10 steps of the pair's magnitudes; bf16: rounded once more."""
    mag = want.abs().amax(-1, keepdim=True) * 2
    bound = 10 * 2.0 ** -24 * mag * 1.01 + HALF[got.dtype] * want.abs() * 1.01
    assert bool(((got.double() - want).abs() <= bound).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits,block", FMT)
@pytest.mark.parametrize("half,page", [(False, 0), (True, 0), (False, 16), (True, 64)])
def test_norm_rope_append(half, page, bits, block, dtype):
    """Ragged tokens of one array of projections, far positions, both layouts of pairs, both permutations."""
    news, lens = [1, 0, 70, 33, 5], [5000, 7, 70, 90, 21]
    cache, pool, q, k, v, w, theta, starts, n, pos, perm, perm_v = write_case(news, lens, 6, 3, bits, block, page, dtype, bits + block + page)
    before = planes(cache)
    out = B.norm_rope_append(cache, q, k, v, starts, n, q_weight=w[0], k_weight=w[1], eps=1e-5, theta=theta, half_split=half,
                             perm_k=perm, perm_v=perm_v, pool=pool)
    check_q(out, rotated64(q, w[0], 1e-5, theta, half, pos))
    check_write(cache, pool, before, rotated64(k, w[1], 1e-5, theta, half, pos), v.double(), news, lens, perm, perm_v, bits, block)
    assert B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("half,page,bits,block,packed", [(False, 64, 4, 32, True), (True, 0, 6, 16, False), (True, 64, 8, 32, True), (False, 0, 4, 128, False)])
@pytest.mark.parametrize("tokens,hq,heads", [(1500, 13, 5), (4000, 13, 5), (2300, 7, 9), (9000, 5, 7), (30001, 6, 3)])
def test_norm_rope_append_runs_of_heads(tokens, hq, heads, half, page, bits, block, packed, dtype):
    """Enough tokens that a warp walks several heads: runs that end inside the queries, cross from them to keys and on to values, odd
    rests, whole tokens; values with a permutation and without."""
    news = [tokens - 1007, 0, 1000, 7]
    lens = [news[0] + 33, 5, 1000, 400]
    cache, pool, q, k, v, w, theta, starts, n, pos, perm, perm_v = write_case(news, lens, hq, heads, bits, block, page, dtype, tokens + bits, packed=packed)
    if not packed:
        perm_v = None
    before = planes(cache)
    out = B.norm_rope_append(cache, q, k, v, starts, n, q_weight=w[0], k_weight=w[1], eps=1e-5, theta=theta, half_split=half, perm_k=perm,
                             perm_v=perm_v, pool=pool)
    check_q(out, rotated64(q, w[0], 1e-5, theta, half, pos))
    check_write(cache, pool, before, rotated64(k, w[1], 1e-5, theta, half, pos), v.double(), news, lens, perm, perm_v, bits, block)
    assert B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("norm,rope", [(False, True), (True, False), (False, False)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm_rope_append_parts(norm, rope, dtype):
    """Without the norm, without the rotation, without both (then the bytes are those of append), no permutations."""
    news, lens = [17, 2], [40, 2]
    cache, pool, q, k, v, w, theta, starts, n, pos, _, _ = write_case(news, lens, 4, 2, 4, 32, 16, dtype, 3, packed=False)
    before = planes(cache)
    kw = dict(q_weight=w[0] if norm else None, k_weight=w[1] if norm else None, eps=0.0, theta=theta if rope else None)
    out = B.norm_rope_append(cache, q, k, v, starts, n, pool=pool, **kw)
    check_q(out, rotated64(q, kw["q_weight"], 0.0, kw["theta"], False, pos))
    check_write(cache, pool, before, rotated64(k, kw["k_weight"], 0.0, kw["theta"], False, pos), v.double(), news, lens, None, None, 4, 32)
    if not norm and not rope:
        assert torch.equal(out, q)
    # queries alone, in place; keys and values alone
    alone = B.norm_rope_append(cache, q, None, None, starts, n, pool=pool, q_out=q, **kw)
    assert alone is q and torch.equal(q, out)
    was = planes(cache)
    for p in (cache.k_mant, cache.k_exp, cache.v_mant, cache.v_exp):
        p[pool.table[1, 0].long()] = 0
    assert B.norm_rope_append(cache, None, k, v, starts, n, pool=pool, **kw) is None
    for now, then in zip(planes(cache), was):
        assert torch.equal(now[pool.table[1, 0].long(), :, :2], then[pool.table[1, 0].long(), :, :2])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm_rope_append_far_ranges(dtype):
    """Rows whose squares leave the fp32 range, or vanish in it, are normalised like any other; rows of zeros give zeros."""
    news, lens = [24], [24]
    cache, pool, q, k, v, w, theta, starts, n, pos, perm, perm_v = write_case(news, lens, 2, 2, 4, 32, 16, dtype, 8)
    for scale, eps in ((2.0 ** 100, 1e-6), (2.0 ** 70, 0.0), (2.0 ** -70, 0.0), (2.0 ** -100, 0.0)):
        x = [(t.float() * scale).to(dtype) for t in (q, k)]
        if eps:
            x[0][3], x[1][5] = 0.0, 0.0
        before = planes(cache)
        out = B.norm_rope_append(cache, x[0], x[1], v.contiguous(), starts, n, q_weight=w[0], k_weight=w[1], eps=eps, theta=theta,
                                 perm_k=perm, perm_v=perm_v, pool=pool)
        check_q(out, rotated64(x[0], w[0], eps, theta, False, pos))
        check_write(cache, pool, before, rotated64(x[1], w[1], eps, theta, False, pos), v.double(), news, lens, perm, perm_v, 4, 32)
    assert B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 8])
def test_norm_rope_append_codes_next_to_borders(bits):
    """A million keys: every code that of the formula in 64 bits, those next to a border too."""
    news, lens = [4096], [100000]
    cols = 100000 // 64 + 1
    perm, perm_v = perms(2, 1)
    g = torch.Generator().manual_seed(7)
    k = torch.randn(4096, 2, D, generator=g).bfloat16().cuda()
    cache = B.Cache(70, 2, D, 64, 32, bits, fill=0)
    table = torch.full((1, cols), -1, dtype=torch.int32)
    first = (100000 - 4096) // 64
    table[0, first:] = torch.arange(cols - first, dtype=torch.int32)
    pool = B.PagePool.of(table.cuda(), None, i32(100000), 70, 64)
    w = 1.0 + 0.2 * torch.randn(D, generator=g).cuda()
    theta = 10000.0 ** (-2.0 * torch.arange(64, dtype=torch.float64, device="cuda") / D)
    pos = torch.arange(100000 - 4096, 100000, device="cuda")
    before = planes(cache)
    B.norm_rope_append(cache, None, k, k, i32(0, 4096), i32(100000), k_weight=w, theta=theta, half_split=True, perm_k=perm, pool=pool)
    check_write(cache, pool, before, rotated64(k, w, 1e-6, theta, True, pos), k.double(), news, lens, perm, None, bits, 32)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("what", ["small keys", "small weights", "large keys"])
def test_norm_rope_append_codes_at_the_ends_of_the_range(what, bits):
    """Keys rotated in the subnormal range, weights there, rows whose norm's factor is there: every code that of the formula."""
    n = 16384
    g = torch.Generator().manual_seed(17)
    k = torch.randn(n, 2, D, generator=g)
    if what == "large keys":
        k = torch.sign(k) * (1.0 + torch.rand(n, 2, D, generator=g)) * 0.999
    scale = {"small keys": 2.0 ** -133, "small weights": 1.0, "large keys": 2.0 ** 126}[what]
    k = (k.bfloat16().double() * scale).float().cuda()
    w = None if what == "small keys" else (1.0 + 0.2 * torch.randn(D, generator=g).cuda()) * (2.0 ** -131 if what == "small weights" else 1.0)
    theta = 10000.0 ** (-2.0 * torch.arange(64, dtype=torch.float64, device="cuda") / D)
    cache = B.Cache(1, 2, D, n, 32, bits, fill=0)
    before = planes(cache)
    B.norm_rope_append(cache, None, k, k, i32(0, n), i32(n), k_weight=w, eps=0.0, theta=theta, half_split=True)
    pos = torch.arange(n, device="cuda")
    check_write(cache, None, before, rotated64(k, w, 0.0, theta, True, pos), k.double(), [n], [n], None, None, bits, 32)
    assert B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("page", [0, 16])
def test_norm_rope_append_flags(page):
    """Positions before the first and behind the cache, missing pages, tokens of no sequence: not stored; q is written for all
    tokens of sequences.  Non-finite keys are flagged."""
    news, lens = [4, 4, 4], [20, 20, 20]
    cache, pool, q, k, v, w, theta, starts, n, pos, perm, perm_v = write_case(news, lens, 2, 2, 4, 32, page, torch.float32, 1)
    kw = dict(q_weight=w[0], k_weight=w[1], theta=theta, pool=pool)
    want = B.norm_rope_append(cache, q, k, v, starts, n, **kw)
    assert B.device_status() == 0
    before = planes(cache)
    bad = i32(2, 20, cache.fmt.max_seq + 3 if pool is None else 35)       # two tokens before the first position | three behind the end
    if pool is not None:
        pool.table[1, 1] = -1
    cache.k_mant[:] = 9
    got = B.norm_rope_append(cache, q, k, v, starts, bad, **kw)
    assert B.device_status() == B.FLAG_POSITION
    assert bool(torch.isfinite(got).all())
    assert torch.equal(got[4:8], want[4:8])
    stored = int((cache.k_mant != 9).any(-1).any(1).sum())
    assert stored == (2 + 4 + 1 if pool is None else 2 + 0 + 1)
    for p, x in zip((cache.k_mant, cache.k_exp, cache.v_mant, cache.v_exp), before):
        p.copy_(x)
    got = torch.full_like(q, 3.0)
    B.norm_rope_append(cache, q, k, v, i32(0, 2, 2, 5), n, q_out=got, **kw)
    assert bool((got[5:] == 3.0).all()) and bool((got[:5] != 3.0).any())
    B.device_status()
    k2 = k.clone()
    k2[1, 0, 5] = math.nan
    B.norm_rope_append(cache, q, k2, v, starts, i32(20, 20, 20) if pool is None else i32(20, 4, 20), **kw)
    assert B.device_status() == B.FLAG_NONFINITE


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [3, 40])
@pytest.mark.parametrize("page", [0, 16])
def test_norm_rope_append_starts_that_decrease(page, batch):
    """Flagged, nothing is stored; the next call is served."""
    news, lens = [3, 60, 2] + [1] * (batch - 3), [100, 60, 80] + [50] * (batch - 3)
    cache, pool, q, k, v, w, theta, starts, n, pos, perm, perm_v = write_case(news, lens, 2, 2, 4, 32, page, torch.bfloat16, 4)
    before, good, rows = planes(cache), starts.tolist(), q.shape[0]
    kw = dict(q_weight=w[0], k_weight=w[1], theta=theta, perm_k=perm, perm_v=perm_v, pool=pool)
    swapped = good[:batch - 1] + [good[batch], good[batch - 1]]
    for bad in ([0, 63, 3] + good[3:], [5, 0] + good[2:], swapped, [0] * batch + [-3], [rows, 0] + [0] * (batch - 1), [0, rows] + [0] * (batch - 1)):
        B.norm_rope_append(cache, q, k, v, i32(*bad), n, **kw)
        down = any(min(max(y, 0), rows) < min(max(x, 0), rows) for x, y in zip(bad, bad[1:]))
        assert B.device_status() == (B.FLAG_POSITION if down else 0), bad
        assert all(torch.equal(x, y) for x, y in zip(planes(cache), before)), bad
    out = B.norm_rope_append(cache, q, k, v, starts, n, **kw)
    check_q(out, rotated64(q, w[0], 1e-6, theta, False, pos))
    check_write(cache, pool, before, rotated64(k, w[1], 1e-6, theta, False, pos), v.double(), news, lens, perm, perm_v, 4, 32)
    assert B.device_status() == 0


# ----------------------------------------------------------------------------------------------- pages
class Model:
    """The pages' bookkeeping step by step."""

    def __init__(self, batch, max_pages, n_pages, page):
        self.table, self.refs, self.lens, self.page = np.full((batch, max_pages), -1), np.zeros(n_pages, int), np.zeros(batch, int), page

    def held(self, n):
        return min(-(-n // self.page), self.table.shape[1])

    def free(self, lo, hi):
        for b, n in enumerate(self.lens):
            for i in range(self.table.shape[1]):
                x = self.table[b, i]
                if x >= 0 and i * self.page >= lo[b] and ((i + 1) * self.page <= hi[b] or hi[b] >= n):
                    self.refs[x] -= 1
                    self.table[b, i] = -1
            if hi[b] >= n:
                self.lens[b] = min(n, max(lo[b], 0))

    def fork(self, src, dst):
        for s, d in zip(src, dst):
            for i in range(self.held(self.lens[s])):
                if self.table[s, i] >= 0:
                    self.table[d, i] = self.table[s, i]
                    self.refs[self.table[s, i]] += 1
            self.lens[d] = self.lens[s]

    def reserve(self, more):
        """Sequence by sequence; free numbers are those from before the call."""
        pairs = np.full((len(self.lens), 2), -1)
        left = [i for i, r in enumerate(self.refs) if r <= 0]
        owners, out, full = self.refs.copy(), [], False
        writers = {}
        for b, n in enumerate(self.lens):
            if more[b] <= 0:
                continue
            first, keeps = False, False
            at = n // self.page
            old = self.table[b, at] if n % self.page and at < self.table.shape[1] else None
            if old is not None:
                if old < 0:
                    first = True
                elif owners[old] > 1:
                    keeps = writers.get(old, 0) >= owners[old] - 1
                    first = not keeps
                    writers[old] = writers.get(old, 0) + 1
            entries = ([at] if first else []) + list(range(self.held(n), self.held(n + more[b])))
            full |= len(entries) > len(left) - len(out)
            if full and (entries or keeps):
                out += [None] * len(entries)
                continue
            for e in entries:
                x = left[len(out)]
                out.append(x)
                if e == at and first and old >= 0:
                    pairs[b] = old, x
                    self.refs[old] -= 1
                self.table[b, e] = x
                self.refs[x] = 1
            self.lens[b] = n + more[b]
        return pairs


def same(pool, model):
    return (np.array_equal(pool.table.cpu().numpy(), model.table) and np.array_equal(pool.refs.cpu().numpy(), model.refs)
            and np.array_equal(pool.lens.cpu().numpy(), model.lens))


@pytest.mark.gpu
@pytest.mark.parametrize("batch,max_pages,n_pages,page", [(5, 9, 40, 16), (64, 33, 3000, 32), (300, 20, 5000, 16), (1024, 4, 9001, 64)])
def test_pages_against_a_model(batch, max_pages, n_pages, page):
    """Random rounds of free, fork, reserve and compact; enough pages."""
    rng = np.random.default_rng(batch)
    pool, model = B.PagePool(batch, max_pages, n_pages, page), Model(batch, max_pages, n_pages, page)
    to = lambda x: torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()
    for step in range(12):
        lo = np.where(rng.random(batch) < 0.4, 0, rng.integers(0, max_pages * page, batch))
        hi = np.where(rng.random(batch) < 0.5, 1 << 30, rng.integers(0, max_pages * page, batch))
        B.pages_free(pool, to(lo), to(hi))
        model.free(lo, hi)
        assert same(pool, model), f"free, step {step}"
        empty = [b for b in range(batch) if model.lens[b] == 0 and (model.table[b] < 0).all()]
        others = [b for b in range(batch) if b not in set(empty)]
        if others and empty:
            dst = rng.permutation(empty)[:max(1, len(empty) // 2)]
            src = rng.choice(others, len(dst))
            B.pages_fork(pool, to(src), to(dst))
            model.fork(src, dst)
            assert same(pool, model), f"fork, step {step}"
        more = np.where(rng.random(batch) < 0.3, -1, rng.integers(0, 3 * page, batch))
        more = np.minimum(more, max_pages * page - model.lens)
        used = int((model.refs > 0).sum())
        if used + batch * 4 > n_pages:
            more[:] = np.minimum(more, 1)
        pairs = B.pages_reserve(pool, to(more))
        assert np.array_equal(pairs.cpu().numpy(), model.reserve(more)), f"pairs, step {step}"
        assert same(pool, model), f"reserve, step {step}"
        if step % 4 == 3:
            check_compact(pool, model)
    flags = B.device_status()
    assert flags in (0, B.FLAG_PAGES)


def check_compact(pool, model):
    """Packed into another pool, then in place."""
    n = len(model.refs)
    used = [i for i in range(n) if model.refs[i] > 0]
    dst = B.PagePool(*pool.table.shape, n + 5, pool.page_tokens)
    dst.refs[:] = 77
    moves, count = B.pages_compact(pool, dst=dst)
    assert int(count) == len(used)
    moves = moves.cpu().numpy()
    assert np.array_equal(moves[:len(used)], np.stack([used, np.arange(len(used))], 1).reshape(-1, 2)) and (moves[len(used):] == -1).all()
    number = np.full(n + 1, -1)
    number[used] = np.arange(len(used))
    assert np.array_equal(dst.table.cpu().numpy(), number[model.table])
    assert np.array_equal(dst.refs.cpu().numpy(), np.concatenate([model.refs[used], np.zeros(n + 5 - len(used), int)]))
    assert np.array_equal(dst.lens.cpu().numpy(), model.lens) and same(pool, model)
    moves, count = B.pages_compact(pool)
    high, holes = [x for x in used if x >= len(used)], [i for i in range(len(used)) if model.refs[i] <= 0]
    assert int(count) == len(high) == len(holes)
    assert np.array_equal(moves.cpu().numpy()[:len(high)], np.array([high, holes]).T.reshape(-1, 2))
    number = np.arange(n + 1)
    number[n] = -1
    number[high] = holes
    model.table = number[model.table]
    for a, b in zip(high, holes):
        model.refs[b], model.refs[a] = model.refs[a], 0
    assert same(pool, model), "compact"


@pytest.mark.gpu
def test_pages_run_out():
    """Too few free pages: sequences before it get theirs, it and those behind it nothing; the table's end."""
    to = lambda *x: i32(*x)
    pool, model = B.PagePool(6, 4, 10, 16), Model(6, 4, 10, 16)
    for more in ([20, 20, 0, 0, 0, 0], [0, 0, 60, 16, 16, 5], [0, 0, 17, 16, 1, 0], [1, 1, 1, 1, 1, 1]):
        pairs = B.pages_reserve(pool, to(*more))
        assert np.array_equal(pairs.cpu().numpy(), model.reserve(np.array(more)))
        assert same(pool, model), more
    assert B.device_status() == B.FLAG_PAGES
    # shared pages when they run out: nobody keeps a page that a refused sequence still has
    for free in range(5):
        pool, model = B.PagePool(5, 2, 1 + free, 16), Model(5, 2, 1 + free, 16)
        for p in (pool, model):
            p.table[0, 0], p.refs[0], p.lens[0] = 0, 1, 5
        B.pages_fork(pool, to(0, 0, 0), to(1, 2, 3))
        model.fork([0, 0, 0], [1, 2, 3])
        pairs = B.pages_reserve(pool, to(2, 2, 2, 2, 0))
        assert np.array_equal(pairs.cpu().numpy(), model.reserve(np.array([2, 2, 2, 2, 0])))
        assert same(pool, model), free
        assert int(pool.lens[3]) == (7 if free >= 3 else 5)
    B.device_status()
    # past the table's end: pages up to there, the length grows, flagged
    pool, model = B.PagePool(2, 3, 10, 16), Model(2, 3, 10, 16)
    for more in ([40, 1], [40, 1], [1, 1]):
        B.pages_reserve(pool, to(*more))
        model.reserve(np.array(more))
        assert same(pool, model)
    assert pool.lens.tolist() == [81, 3] and B.device_status() == B.FLAG_PAGES
    # a destination with too few pages
    dst = B.PagePool(2, 3, 2, 16)
    moves, count = B.pages_compact(pool, dst=dst)
    assert int(count) == 2 and B.device_status() == B.FLAG_PAGES
    assert int((dst.table >= 0).sum()) == 2 and dst.refs.tolist() == [1, 1]


@pytest.mark.gpu
@pytest.mark.parametrize("few", [0, 3])
def test_pages_reserve_counts_past_32_bits(few):
    """1024 sequences that ask for some 2^31 pages between them: those that find pages get them, the others stay as they were."""
    pool = B.PagePool(1024, 1 << 21, 100, 16)
    more = torch.full((1024,), 1 << 25, dtype=torch.int32, device="cuda")
    more[:few] = 17
    pairs = B.pages_reserve(pool, more)
    want = torch.zeros(1024, dtype=torch.int32, device="cuda")
    want[:few] = 17
    assert torch.equal(pool.lens, want)
    assert pool.table[:few, :2].flatten().tolist() == list(range(2 * few))
    assert int((pool.table >= 0).sum()) == 2 * few and int(pool.refs.sum()) == 2 * few
    assert bool((pairs == -1).all()) and B.device_status() == B.FLAG_PAGES


@pytest.mark.gpu
def test_pages_fork_skips_what_it_must():
    pool = B.PagePool(6, 2, 12, 16)
    B.pages_reserve(pool, i32(20, 5, 0, 0, 0, 0))
    was = pool.table.clone(), pool.refs.clone(), pool.lens.clone()
    # taken, out of range, from one that is being made, negative source
    B.pages_fork(pool, i32(0, 0, 7, 0, -1), i32(1, 9, 2, -1, 3))
    assert all(torch.equal(a, b) for a, b in zip(was, (pool.table, pool.refs, pool.lens)))
    assert B.device_status() == B.FLAG_POSITION
    B.pages_fork(pool, i32(0, 1, 2), i32(2, 2, 4))              # 2 named twice, and the source of another: the rest goes
    assert pool.lens.tolist() == [20, 5, 20, 0, 0, 0] and B.device_status() == B.FLAG_POSITION
    assert torch.equal(pool.table[2], pool.table[0]) and pool.refs[pool.table[0].long()].tolist() == [2, 2]


@pytest.mark.gpu
@pytest.mark.parametrize("bits,block,page", [(4, 32, 16), (6, 128, 64), (8, 16, 32), (4, 128, 256)])
def test_pages_copy(bits, block, page):
    src, dst = B.Cache(9, 3, D, page, block, bits), B.Cache(12, 3, D, page, block, bits, fill=1)
    fill(src, bits)
    names = ("k_mant", "k_exp", "v_mant", "v_exp")
    want = {n: getattr(dst, n).clone() for n in names}
    pairs = i32(3, 11, -1, 2, 8, 0, 9, 4, 2, 12, 0, 5, 4, -1, 1, 1).reshape(8, 2)
    for n in names:
        want[n][11], want[n][0], want[n][5] = getattr(src, n)[3], getattr(src, n)[8], getattr(src, n)[0]
    B.pages_copy(src, pairs, count=i32(7), dst=dst)
    for n in names:
        assert torch.equal(getattr(dst, n), want[n])
    assert B.device_status() == B.FLAG_POSITION          # numbers outside the pools
    B.pages_copy(dst, i32(11, 7).reshape(1, 2))
    for n in names:
        want[n][7] = want[n][11]
        assert torch.equal(getattr(dst, n), want[n])
    B.pages_copy(dst, i32(0, 1).reshape(1, 2), count=i32(0))
    B.pages_copy(dst, torch.empty(0, 2, dtype=torch.int32, device="cuda"))
    assert torch.equal(dst.k_mant, want["k_mant"]) and B.device_status() == 0


# ----------------------------------------------------------------------------------------------- together
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,bits", [(torch.bfloat16, 4), (torch.float32, 8)])
def test_serving_loop(dtype, bits):
    """Prompts written and attended, branches forked, tokens decoded, a branch dropped, the pool packed, in two layers that
    share the table: every attention against the reference on a contiguous cache that gets the same tokens by append."""
    H, G, P, layers = 2, 2, 32, 2
    g = torch.Generator().manual_seed(1)
    pool = B.PagePool(4, 8, 26, P)
    caches = [B.Cache(26, H, D, P, 32, bits) for _ in range(layers)]
    w = [1.0 + 0.2 * torch.randn(D, generator=g).cuda() for _ in range(2)]
    theta = 10000.0 ** (-2.0 * torch.arange(64, dtype=torch.float64, device="cuda") / D)
    perm, perm_v = perms(H, 5)
    kept = [[[] for _ in range(4)] for _ in range(layers)]             # rotated keys and values of every sequence, fp64

    def step(news):
        more = i32(*news)
        pairs = B.pages_reserve(pool, more)
        starts = i32(*np.concatenate([[0], np.cumsum(news)]).tolist())
        lens = pool.lens.tolist()
        pos = torch.cat([torch.arange(n - m, n) for n, m in zip(lens, news)]).cuda()
        for li, cache in enumerate(caches):
            B.pages_copy(cache, pairs)
            x = torch.randn(sum(news), H * (G + 2), D, generator=g).to(dtype).cuda()
            q, k, v = x[:, :H * G], x[:, H * G:H * (G + 1)], x[:, H * (G + 1):]
            qr = B.norm_rope_append(cache, q, k, v, starts, pool.lens, q_weight=w[0], k_weight=w[1], theta=theta, half_split=True,
                                    perm_k=perm, perm_v=perm_v, pool=pool)
            got = B.ragged_attn(cache, qr, starts, pool.lens, max(news), window=90, n_sink=4, perm_k=perm,
                                inv_perm_v=inverse(perm_v), pool=pool)
            check(got, *reference(cache, pool, qr, news, lens, perm, perm_v, 90, 4))
            k64 = rotated64(k, w[1], 1e-6, theta, True, pos)
            row = 0
            for b, m in enumerate(news):
                for i in range(m):
                    kept[li][b].append((k64[row + i], v[row + i].double()))
                row += m
        assert B.device_status() == 0

    def agree():
        """Every cached row is the cast of the token that was written there."""
        for li, cache in enumerate(caches):
            for b, n in enumerate(pool.lens.tolist()):
                assert n == len(kept[li][b])
                if n == 0:
                    continue
                for which, pm, j in (("k", perm, 0), ("v", perm_v, 1)):
                    want = torch.stack([t[j] for t in kept[li][b]]).gather(-1, pm.long()[None].expand(n, H, D))
                    m, e = cast64(want, bits, 32)
                    t = torch.arange(n, device="cuda")
                    pg, rw = pool.table[b, t // P].long(), t % P
                    assert np.array_equal(fields(getattr(cache, which + "_mant")[pg, :, rw], bits), m)
                    assert np.array_equal(getattr(cache, which + "_exp")[pg, :, rw].cpu().numpy(), e)

    def fork(src, dst):
        B.pages_fork(pool, i32(*src), i32(*dst))
        for s, d in zip(src, dst):
            for li in range(layers):
                kept[li][d] = list(kept[li][s])

    def cut(lo):
        B.pages_free(pool, lo=i32(*lo))
        for li in range(layers):
            kept[li] = [x[:n] for x, n in zip(kept[li], lo)]

    step([100, 37, 0, 0])
    agree()
    fork([0, 1], [2, 3])
    step([1, 1, 1, 1])
    step([1, 3, 1, 20])
    agree()
    cut([10 ** 6, 30, 0, 10 ** 6])
    fork([3], [2])
    step([5, 40, 1, 1])
    agree()
    moves, count = B.pages_compact(pool)
    for cache in caches:
        B.pages_copy(cache, moves, count=count)
    agree()
    step([1, 1, 1, 1])
    used = int((pool.refs > 0).sum())
    small = B.PagePool(4, 8, used + 4, P)
    moves, count = B.pages_compact(pool, dst=small)
    for li in range(layers):
        to = B.Cache(used + 4, H, D, P, 32, bits)
        B.pages_copy(caches[li], moves, count=count, dst=to)
        caches[li] = to
    pool = small
    agree()
    step([2, 1, 1, 1])
    agree()


@pytest.mark.gpu
def test_graph_of_a_decode_step():
    """Reserve, copy, write and attend captured once and replayed: lengths grow on the device."""
    H, G, P = 2, 4, 16
    news = [1, 1, 1]
    g = torch.Generator().manual_seed(3)
    perm, perm_v = perms(H, 5)
    make = lambda: paged([40, 3, 17], H, P, 4, 32, 2, perm, perm_v, extra=20, cols=8)
    x = [torch.randn(3, H * (G + 2), D, generator=g).bfloat16().cuda() for _ in range(20)]
    theta = 10000.0 ** (-2.0 * torch.arange(64, dtype=torch.float64, device="cuda") / D)
    starts, more, live = i32(0, 1, 2, 3), i32(1, 1, 1), x[0].clone()
    kw = dict(perm_k=perm, perm_v=perm_v)

    def step(cache, pool, ws, out):
        pairs = B.pages_reserve(pool, more)
        B.pages_copy(cache, pairs)
        q = B.norm_rope_append(cache, live[:, :H * G], live[:, H * G:H * (G + 1)], live[:, H * (G + 1):], starts, pool.lens,
                               theta=theta, pool=pool, **kw)
        B.ragged_attn(cache, q, starts, pool.lens, 1, window=30, n_sink=2, perm_k=perm, inv_perm_v=inverse(perm_v), pool=pool, out=out,
                      workspace=ws)

    cache, pool = make()
    ws = torch.empty(B.ragged_workspace_bytes(cache.fmt, 3, H * G, 1), dtype=torch.uint8, device="cuda")
    out = torch.empty(3, H * G, D, dtype=torch.bfloat16, device="cuda")
    eager = []
    for i in range(20):
        live.copy_(x[i])
        step(cache, pool, ws, out)
        eager.append(out.clone())
    cache2, pool2 = make()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(cache2, pool2, ws, out)
    for i in range(20):
        live.copy_(x[i])
        graph.replay()
        assert torch.equal(out, eager[i]), i
    assert torch.equal(pool.table, pool2.table) and torch.equal(cache.k_mant[pool.table[0, :3].long()], cache2.k_mant[pool.table[0, :3].long()])
    assert B.device_status() == 0


@pytest.mark.gpu
def test_ragged_attn_on_streams_at_once():
    """Four calls with workspaces of their own on four streams give what they give alone."""
    news, lens = [1, 200, 30], [3000, 900, 400]
    args = batch_of(news, lens, 4, 2, 4, 32, 64, torch.bfloat16, 12)
    alone = attend(args, news, window=700, n_sink=4)
    streams = [torch.cuda.Stream() for _ in range(4)]
    outs = []
    torch.cuda.synchronize()
    for _ in range(5):
        for s in streams:
            outs.append(attend(args, news, window=700, n_sink=4, stream=s))
    torch.cuda.synchronize()
    assert all(torch.equal(alone, o) for o in outs)


# ----------------------------------------------------------------------------------------------- refusals (no GPU)
def structs(page=16, n_pages=8, **kw):
    f = B.Format(n_pages, kw.pop("heads", 2), 128, page, kw.pop("block", 32), kw.pop("bits", 4))
    cs = B.CacheStruct(f, 0x10000, 0x20000, 0x30000, 0x40000)
    a = dict(batch=3, max_pages=4, n_pages=n_pages, page_tokens=page, table=0x50000, refs=0x60000, lens=0x70000)
    a.update(kw)
    return f, cs, B.PagesStruct(*a.values())


def test_pages_refusals():
    L = B.lib()
    vp = C.c_void_p
    before = B.launch_count()
    free = lambda ps: L.kvbfp_pages_free(None if ps is None else C.byref(ps), None, None, None)
    assert free(None) == B.ERR_INVALID_ARG
    for bad, rc in ((dict(table=None), B.ERR_INVALID_ARG), (dict(refs=None), B.ERR_INVALID_ARG), (dict(lens=None), B.ERR_INVALID_ARG),
                    (dict(batch=0), B.ERR_INVALID_ARG), (dict(max_pages=0), B.ERR_INVALID_ARG), (dict(page_tokens=48), B.ERR_UNSUPPORTED),
                    (dict(page_tokens=8), B.ERR_UNSUPPORTED), (dict(page_tokens=2048), B.ERR_UNSUPPORTED), (dict(batch=1025), B.ERR_UNSUPPORTED),
                    (dict(max_pages=1 << 27), B.ERR_UNSUPPORTED), (dict(table=0x50004), B.ERR_ALIGNMENT), (dict(refs=0x60008), B.ERR_ALIGNMENT)):
        ps = structs(**bad)[2]
        assert free(ps) == rc, bad
        assert L.kvbfp_pages_workspace_bytes(C.byref(ps)) == 0
    _, cs, ps = structs()
    P = C.byref(ps)
    assert L.kvbfp_pages_fork(P, None, vp(16), 1, None) == B.ERR_INVALID_ARG
    assert L.kvbfp_pages_fork(P, vp(16), vp(16), -1, None) == B.ERR_INVALID_ARG
    assert L.kvbfp_pages_fork(P, vp(16), vp(16), 65536, None) == B.ERR_UNSUPPORTED
    assert L.kvbfp_pages_fork(P, None, None, 0, None) == B.OK
    assert L.kvbfp_pages_reserve(P, None, vp(16), None) == B.ERR_INVALID_ARG
    assert L.kvbfp_pages_reserve(P, vp(16), None, None) == B.ERR_INVALID_ARG
    assert L.kvbfp_pages_reserve(P, vp(16), vp(24), None) == B.ERR_ALIGNMENT
    need = L.kvbfp_pages_workspace_bytes(P)
    compact = lambda a=ps, d=None, mv=16, ct=16, ws=16, n=need: L.kvbfp_pages_compact(
        C.byref(a), C.byref(a if d is None else d), vp(mv), vp(ct), vp(ws), n, None)
    assert compact(mv=None) == B.ERR_INVALID_ARG and compact(ct=None) == B.ERR_INVALID_ARG
    assert compact(ws=None) == B.ERR_WORKSPACE and compact(n=need - 1) == B.ERR_WORKSPACE
    assert compact(ws=24) == B.ERR_ALIGNMENT
    other = structs(table=0x150000, refs=0x160000, lens=0x170000)[2]
    for change in (dict(batch=2), dict(max_pages=5), dict(page_tokens=32), dict(refs=ps.refs), dict(lens=ps.lens), dict(table=0x50000 + 16),
                   dict(refs=0x60000 + 16), dict(table=ps.refs + 16)):
        d = B.PagesStruct(*[change.get(n, getattr(other, n)) for n, _ in B.PagesStruct._fields_])
        assert compact(d=d) == B.ERR_INVALID_ARG, change
    d = B.PagesStruct(*[getattr(ps, n) if n != "n_pages" else 9 for n, _ in B.PagesStruct._fields_])
    assert compact(d=d) == B.ERR_INVALID_ARG               # in place with another number of pages
    copy = lambda a, b, pr=16, n=1: L.kvbfp_pages_copy(C.byref(a), C.byref(b), vp(pr), n, None, None)
    assert L.kvbfp_pages_copy(None, C.byref(cs), vp(16), 1, None, None) == B.ERR_INVALID_ARG
    assert copy(cs, cs, pr=None) == B.ERR_INVALID_ARG and copy(cs, cs, n=-1) == B.ERR_INVALID_ARG
    assert copy(cs, cs, pr=24) == B.ERR_ALIGNMENT and copy(cs, cs, n=0) == B.OK
    for kw in (dict(page=32), dict(bits=8), dict(block=64), dict(heads=3)):
        o = B.CacheStruct(structs(**kw)[0], 0x110000, 0x120000, 0x130000, 0x140000)
        assert copy(cs, o) == B.ERR_INVALID_ARG, kw
    assert copy(cs, B.CacheStruct(cs.fmt, 0x10000 + 1024, 0x120000, 0x130000, 0x140000)) == B.ERR_INVALID_ARG       # overlapping
    assert copy(cs, B.CacheStruct(cs.fmt, 0x110000, 0x10000, 0x130000, 0x140000)) == B.ERR_INVALID_ARG              # one plane in common
    assert copy(cs, B.CacheStruct(cs.fmt, 0x110000, 0x120000, None, 0x140000)) == B.ERR_INVALID_ARG
    assert B.launch_count() == before


def test_write_refusals():
    L = B.lib()
    vp = C.c_void_p
    before = B.launch_count()
    f, cs, ps = structs()
    A = 1 << 24

    def call(cache=cs, pages=ps, q=A, qs=512, k=2 * A, ks=256, v=3 * A, vs=256, dt=1, hq=4, n=5, st=16, ln=16, qw=None, kw=None, eps=1e-6,
             th=None, pk=None, pv=None, out=4 * A):
        return L.kvbfp_norm_rope_append(None if cache is None else C.byref(cache), None if pages is None else C.byref(pages), vp(q), qs,
                                        vp(k), ks, vp(v), vs, dt, hq, n, vp(st), vp(ln), vp(qw), vp(kw), eps, vp(th), 0, vp(pk), vp(pv),
                                        vp(out), None)
    inv = (dict(cache=None), dict(q=None), dict(out=None), dict(k=None), dict(v=None), dict(q=None, k=None, v=None, out=None), dict(st=None),
           dict(ln=None), dict(dt=3), dict(n=-1), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(hq=0), dict(qs=511), dict(ks=128), dict(vs=0),
           dict(out=A + 16), dict(out=2 * A), dict(out=3 * A + 256), dict(out=A, qs=1024), dict(cache=B.CacheStruct(f, 0x10000, 0x20000, None, 0x40000)),
           dict(pages=structs(n_pages=9)[2]), dict(pages=structs(page=32)[2]), dict(pages=structs(table=None)[2]))
    for kw in inv:
        assert call(**kw) == B.ERR_INVALID_ARG, kw
    for kw in (dict(q=A + 8), dict(k=2 * A + 8), dict(out=4 * A + 8), dict(qs=516), dict(ks=257), dict(th=20), dict(qw=18), dict(pk=24), dict(pv=24)):
        assert call(**kw) == B.ERR_ALIGNMENT, kw
    for kw in (dict(n=1 << 27), dict(hq=5000, qs=5000 * 128), dict(pages=structs(page_tokens=48)[2])):
        assert call(**kw) == B.ERR_UNSUPPORTED, kw
    assert call(n=0) == B.OK and call(n=0, out=A) == B.OK and call(n=0, q=None, out=None, hq=0) == B.OK
    assert B.launch_count() == before


def test_ragged_refusals():
    L = B.lib()
    vp = C.c_void_p
    before = B.launch_count()
    f, cs, ps = structs()
    need = L.kvbfp_ragged_workspace_bytes(C.byref(f), 3, 4, 5)
    assert need > 0
    for kw in (dict(batch=0), dict(batch=1025), dict(hq=3), dict(hq=18), dict(hq=0), dict(n=-1)):
        a = dict(batch=3, hq=4, n=5)
        a.update(kw)
        assert L.kvbfp_ragged_workspace_bytes(C.byref(f), a["batch"], a["hq"], a["n"]) == 0, kw

    def call(cache=cs, pages=ps, q=16, dt=1, hq=4, n=5, batch=3, st=16, ln=16, new=1, window=0, sink=0, pk=None, iv=None, scale=0.0, out=16, ws=16,
             size=need):
        return L.kvbfp_ragged_attn(None if cache is None else C.byref(cache), None if pages is None else C.byref(pages), vp(q), dt, hq, n,
                                   batch, vp(st), vp(ln), new, window, sink, vp(pk), vp(iv), scale, vp(out), vp(ws), size, None)
    for kw in (dict(cache=None), dict(q=None), dict(st=None), dict(ln=None), dict(out=None), dict(dt=2), dict(hq=3), dict(hq=0), dict(n=-1), dict(batch=2),
               dict(new=-1), dict(window=-1), dict(sink=-1), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(pages=None),
               dict(pages=structs(n_pages=9)[2]), dict(cache=B.CacheStruct(f, None, 0x20000, 0x30000, 0x40000))):
        assert call(**kw) == B.ERR_INVALID_ARG, kw
    for kw in (dict(q=24), dict(out=24), dict(ws=24), dict(pk=24), dict(iv=24)):
        assert call(**kw) == B.ERR_ALIGNMENT, kw
    assert call(hq=18) == B.ERR_UNSUPPORTED and call(n=1 << 27) == B.ERR_UNSUPPORTED
    assert call(ws=None) == B.ERR_WORKSPACE and call(size=need - 1) == B.ERR_WORKSPACE
    assert call(n=0) == B.OK
    assert B.launch_count() == before


def test_calls_without_tokens():
    """No new tokens: arrays without an address are no error, everything else is checked all the same."""
    L = B.lib()
    vp = C.c_void_p
    before = B.launch_count()
    f, cs, ps = structs()
    need = L.kvbfp_ragged_workspace_bytes(C.byref(f), 3, 4, 0)

    def write(n=0, st=16, ln=16, q=None, out=None, dt=1, pages=ps):
        return L.kvbfp_norm_rope_append(C.byref(cs), C.byref(pages), vp(q), 512, None, 256, None, 256, dt, 4, n, vp(st), vp(ln), None, None, 1e-6,
                                        None, 0, None, None, vp(out), None)

    def attend(n=0, st=16, ln=16, q=None, out=None, dt=1, ws=16, new=0):
        return L.kvbfp_ragged_attn(C.byref(cs), C.byref(ps), vp(q), dt, 4, n, 3, vp(st), vp(ln), new, 0, 0, None, None, 0.0, vp(out), vp(ws), need, None)
    for call in (write, attend):
        assert call() == B.OK and call(q=16) == B.OK and call(out=16) == B.OK
        for kw in (dict(n=1), dict(n=-1), dict(st=None), dict(ln=None), dict(dt=3)):
            assert call(**kw) == B.ERR_INVALID_ARG, kw
        assert call(q=24) == B.ERR_ALIGNMENT
    assert attend(new=-1) == B.ERR_INVALID_ARG and attend(ws=None) == B.ERR_WORKSPACE
    assert write(pages=structs(n_pages=9)[2]) == B.ERR_INVALID_ARG
    assert B.launch_count() == before


@pytest.mark.gpu
@pytest.mark.parametrize("page", [0, 16])
def test_steps_without_tokens(page):
    """A step in which no sequence has new tokens, as a loop over steps makes it."""
    cache, pool, _, _, n, perm, perm_v = batch_of([0, 0], [5, 40], 2, 2, 4, 32, page, torch.bfloat16, 1)
    starts, before = i32(0, 0, 0), planes(cache)
    for q in (torch.empty(0, 4, D, dtype=torch.bfloat16, device="cuda"), torch.empty(3, 8, D, dtype=torch.bfloat16, device="cuda")[:0, :4]):
        k = torch.empty(0, 2, D, dtype=torch.bfloat16, device="cuda")
        for args in ((q, k, k), (q, None, None), (None, k, k)):
            got = B.norm_rope_append(cache, *args, starts, n, perm_k=perm, perm_v=perm_v, pool=pool)
            assert got is None if args[0] is None else got.shape == q.shape
        assert B.ragged_attn(cache, q, starts, n, 0, perm_k=perm, pool=pool).shape == q.shape
    assert all(torch.equal(x, y) for x, y in zip(planes(cache), before))
    assert B.device_status() == 0


@pytest.mark.parametrize("batch,most", [(512, 1 << 23), (1024, 1 << 26), (3, 1 << 30)])
def test_ragged_workspace_of_long_batches(batch, most):
    """Batches whose tokens pass 32 bits: as much as the most that a call takes."""
    f = structs()[0]
    assert B.ragged_workspace_bytes(f, batch, 4, most) == B.ragged_workspace_bytes(f, batch, 4, (1 << 26) // batch) > 0


class Plane:
    """What Cache.of looks at of a plane (no second device is needed)."""
    dtype, is_cuda = torch.uint8, True

    def __init__(self, shape, device):
        self.shape, self.device = shape, device

    def is_contiguous(self):
        return True

    def get_device(self):
        return self.device


@pytest.mark.parametrize("at", range(4))
def test_cache_of_planes_on_two_devices(at):
    """Calls look at the first plane's device: planes elsewhere are refused when the cache is put together."""
    shapes = [(5, 2, 16, w) for w in (64, 4, 64, 4)]
    assert B.Cache.of(*(Plane(s, 0) for s in shapes), 32, 4).fmt.head_dim == D
    with pytest.raises(ValueError):
        B.Cache.of(*(Plane(s, int(i == at)) for i, s in enumerate(shapes)), 32, 4)
