"""The paged cache where it can go wrong: scales of the smallest sizes, batches of more prompts than one call takes, prefills that do not fit,
how exact the shared rows are, calls one behind the other; against plain float64 forms."""
import math
import os
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import paper_2404_09529_b200 as pp
from paper_2404_09529_b200.runner import PagedCaches, PagedDecoder, PrefillBatch
from test_paged import BF16, E4M3, Pages, check_step, host64, new_rows, normal, rotate64, shared_case


# ------------------------------------------------------------------------------------------
# 8-bit pages: scales of the smallest sizes
# ------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("fresh", [True, False])
@pytest.mark.parametrize("hq,hkv,d", [(8, 4, 128), (6, 2, 64)])
@pytest.mark.parametrize("k_scale", [0.02, 1e-9, 2e-15, 1e-30, 2.0 ** -126])
def test_8_bit_step_of_queries_of_zeros(k_scale, hq, hkv, d, fresh):
    """Queries of zeros, tiny ones and ordinary ones over keys whose scale may be any: all scores are next to 0, so O is next to the mean
    of the values, whatever part of a unit of rows the prompt's last rows fill."""
    lengths = np.array([1, 2, 15, 17, 31, 33, 64, 100, 129, 500], np.int32)
    P = Pages(lengths + fresh, hkv, d, 16, False, E4M3, seed=d)
    P.k_scale = torch.full((hkv,), k_scale, dtype=torch.float32)
    P.poison(lengths)
    caches = P.cuda()
    q, k, v = new_rows(len(lengths), hq, hkv, d, 3, False)
    q[:, 0] = 0
    q[:, 1] = (q[:, 1].float() * 2.0 ** -110).to(BF16)
    q[:5, 2] = 0
    args = (k, v) if fresh else (None, None)
    before = [x.clone() for x in P.pools]
    dec = PagedDecoder(caches, hq, 10000.0)
    out = dec.step(torch.from_numpy(lengths).cuda(), q, *args)
    assert dec.device_status() == 0
    check_step(P, lengths, q, *args, out, before, 10000.0)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,prompts", [(4, 1, 128, 1100), (2, 2, 64, 600), (8, 1, 128, 3)])
@pytest.mark.parametrize("v_scale", [0.02, 2e-15, 2.0 ** -118, 2.0 ** -124])
def test_8_bit_step_over_values_of_a_small_scale(v_scale, hq, hkv, d, prompts):
    """Queries of zeros, so that O is the mean of the values and sums of weights are as large as they get, over values whose scale may be any;
    many prompts, each the work of one warp, and a few, whose parts are joined."""
    lengths = np.random.default_rng(d).integers(200, 500, prompts).astype(np.int32)
    P = Pages(lengths, hkv, d, 64, True, E4M3, seed=d + hq)
    P.v_scale = torch.full((hkv,), v_scale, dtype=torch.float32)
    caches = P.cuda()
    dec = PagedDecoder(caches, hq, 10000.0)
    got = host64(dec.step(torch.from_numpy(lengths).cuda(), torch.zeros(prompts, hq, d, dtype=BF16, device="cuda")))
    assert dec.device_status() == 0
    for i, n in enumerate(int(x) for x in lengths):
        values = P.rows(1, i, n)
        want, mean = (np.repeat(x.mean(0), hq // hkv, 0) for x in (values, np.abs(values)))
        # Weights are 1. Sums in fp32, twice 2^-24 a term for tensor cores that truncate, and a few roundings behind them; then half of
        # a step of bf16: 2^-8 of O, or 2^-134 where bf16 has no bits for more.
        assert (np.abs(got[i] - want) <= (n + 16) * 2.0 ** -23 * mean + np.abs(want) * 2.0 ** -8 + 2.0 ** -134).all(), i


# ------------------------------------------------------------------------------------------
# Appending: rows whose heads go round a block's loop
# ------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("hkv,d,dtype,fused,rotated", [
    (32, 128, BF16, True, False), (40, 128, E4M3, False, False), (33, 128, BF16, False, True), (48, 64, E4M3, True, False),
])
def test_append_of_many_wide_rows_is_that_of_few(hkv, d, dtype, fused, rotated):
    """A row of more than 2048 elements is shared out to several blocks while few are appended, and is the work of one where there are
    many: the same bits."""
    rows, prompts, page = 1300, 7, 32
    rng = np.random.default_rng(hkv)
    prompt = rng.integers(-1, prompts, rows).astype(np.int32)
    position = np.arange(rows, dtype=np.int32)         # (every cell once)
    s = torch.full((hkv,), 0.03, device="cuda") if dtype == E4M3 else None
    many, few = (PagedCaches.allocate(prompts, prompts * -(-rows // page), rows, hkv, d, page, dtype=dtype, k_scale=s, v_scale=s) for _ in range(2))
    for c in (many, few):
        for i in range(prompts):
            c.reserve(i, rows)
    prompt, position = (torch.from_numpy(x).cuda() for x in (prompt, position))
    _, k, v = new_rows(rows, 1, hkv, d, 8, fused)
    many.append(prompt, position, k, v, 10000.0, rotated=rotated)
    for a in range(0, rows, 100):
        few.append(prompt[a:a + 100], position[a:a + 100], k[a:a + 100], v[a:a + 100], 10000.0, rotated=rotated)
    assert int(many.status) == int(few.status) == 0 and torch.equal(many.page_table, few.page_table)
    raw = torch.uint8 if dtype == E4M3 else torch.int16
    for a, b in ((many.k_pages, few.k_pages), (many.v_pages, few.v_pages)):
        assert torch.equal(a.view(raw), b.view(raw)) and bool(a.view(raw).any())


# ------------------------------------------------------------------------------------------
# How exact the shared rows are
# ------------------------------------------------------------------------------------------
# Queries reach the products as two bf16 numbers each, 2^-16, their weights as one.
def attend_shared(q, keys, values, scale):
    """O [heads, d] of queries of one KV head, and how far it may be off. e: what a score may be off by, from the query's parts, its
    rotation in fp32 (3 roundings) and a sum of 2 d products in fp32, twice that for tensor cores that truncate; a weight over their sum
    is then off by a factor of exp(2 e) at most, and by 2^-8 as one bf16 number, 2^-22 of its exponential and n 2^-23 of the sums. All of
    it times sum p |v|, and the last rounding, 2^-8 of O."""
    s = keys @ q.T * scale                             # [n, heads]
    p = np.exp(s - s.max(0))
    p /= p.sum(0)
    o, mean = p.T @ values, p.T @ np.abs(values)
    size = (np.abs(keys) @ np.abs(q).T).max(0) * abs(scale)
    d, n = q.shape[1], len(keys)
    e = size * (2.0 ** -16 + (4 * d + 8) * 2.0 ** -24) + 2.0 ** -22
    err = mean * (np.exp(2 * e) - 1 + 2.0 ** -8 + n * 2.0 ** -23 + 64 * 2.0 ** -23)[:, None]
    return o, np.abs(o) * 2.0 ** -8 + err * (1 + 2.0 ** -8)


@pytest.mark.gpu
@pytest.mark.parametrize("samples,hq,hkv,d,page", [(5, 4, 4, 64, 16), (40, 8, 1, 64, 32), (16, 8, 1, 128, 16), (3, 2, 2, 128, 64), (48, 16, 2, 128, 16)])
def test_queries_over_shared_rows_keep_their_lower_part(samples, hq, hkv, d, page):
    """Keys whose products with the queries cancel but for what a query loses as one bf16 number: k = +-c (q~_b, -q~_a) at elements
    a and b, with q~ the rounded query. The scores are then +-1 to +-4 with both parts and 0 with one."""
    shared, n = 512, 520
    P, lengths, g = shared_case([(shared, [n] * samples)], hq, hkv, d, page, False, False, seed=d + samples, poison=False)
    rng = np.random.default_rng(samples)
    raw = torch.from_numpy(rng.standard_normal((hkv, d))).to(BF16)
    turned = rotate64(host64(raw)[None], [n - 1], 10000.0)[0]
    rounded = host64(torch.from_numpy(turned).float().to(BF16))
    scale, sign = 1 / math.sqrt(d), np.where(rng.random(shared) < 0.5, -1.0, 1.0)
    ids = torch.from_numpy(P.table[0, :shared // page].astype(np.int64))
    keys = torch.from_numpy(0.05 * rng.standard_normal((shared, hkv, d)))
    values = torch.from_numpy(0.1 * rng.standard_normal((shared, hkv, d)) + sign[:, None, None])
    for h in range(hkv):
        cross = np.outer(turned[h], rounded[h]) - np.outer(rounded[h], turned[h])      # q_a q~_b - q_b q~_a
        a, b = np.unravel_index(np.abs(cross).argmax(), cross.shape)
        c = 2.0 ** np.ceil(np.log2(1 / (abs(cross[a, b]) * scale)))                    # scores of 1 to 2
        keys[:, h, [a, b]] = torch.from_numpy(np.outer(sign, 2 * c * np.array([rounded[h, b], -rounded[h, a]])))
    for pool, rows in zip(P.pools, (keys, values)):
        pool[ids] = rows.to(BF16).view(-1, page, hkv, d).transpose(1, 2)
    caches = P.cuda()
    q = raw.repeat_interleave(hq // hkv, 0).expand(samples, hq, d).contiguous().cuda()
    dec = PagedDecoder(caches, hq, 10000.0)
    got = host64(dec.step(torch.from_numpy(lengths).cuda(), q, groups=g))
    assert dec.device_status() == 0
    for i in range(samples):
        k, v = (P.rows(w, i, n) for w in (0, 1))
        for h in range(hkv):
            per = hq // hkv
            o, tol = attend_shared(turned[h][None], k[:, h], v[:, h], scale)
            lossy = attend_shared(rounded[h][None], k[:, h], v[:, h], scale)[0]
            assert (np.abs(o - lossy) > 4 * tol).mean() > 0.9          # (a query of one part would be seen)
            for m in range(per):
                assert (np.abs(got[i, h * per + m] - o[0]) <= tol[0]).all(), (i, h, m)


@pytest.mark.gpu
@pytest.mark.parametrize("groups,hq,hkv,d,page,softmax_scale,outside", [
    ([(320 + 64 * g, [700 + 3 * i + g for i in range(8)]) for g in range(5)], 32, 32, 128, 64, 0.0, ()),      # 1280 query heads: a warp joins each
    ([(1000, [1000 + i for i in range(40)])], 32, 8, 128, 16, 0.05, (3, -1, 0, 200)),                         # 160 query rows of a KV head
    ([(256, [256 + i for i in range(17)])], 8, 1, 128, 128, 0.0, ()),                                         # 136 rows: a second tile of 8
    ([(256, [300] * 16), (512, [513, -1, 600])], 8, 1, 128, 32, 0.2, ()),
    ([(2000, [2100 + i for i in range(33)])], 8, 1, 128, 16, 0.0, ()),                                        # 264 rows: both tiles, and a split item of 8
    ([(512, [520 + i for i in range(40)]), (48, [60] * 3)], 8, 2, 64, 16, 0.25, (77,)),
    ([(0, [20] * 20), (300, [310, 305, 420])], 8, 1, 128, 16, 0.0, ()),                                       # 160 rows that share nothing
    ([(128, [130] * 40), (16, [30] * 2), (2100, [2200] * 2)], 8, 1, 128, 16, 0.0, (1,)),                      # one key tile; items of both kinds
])
def test_shared_step_within_its_roundings(groups, hq, hkv, d, page, softmax_scale, outside):
    """Every element of O within what the roundings that there are can do, at the softmax scales that a model may have."""
    P, lengths, g = shared_case(groups, hq, hkv, d, page, True, False, seed=hq + d, outside=outside)
    caches = P.cuda()
    q = new_rows(len(lengths), hq, hkv, d, 31, True)[0]
    dec = PagedDecoder(caches, hq, 10000.0, softmax_scale=softmax_scale)
    got = host64(dec.step(torch.from_numpy(lengths).cuda(), q, groups=g))
    assert dec.device_status() == 0
    per = hq // hkv
    for i, n in enumerate(int(x) for x in lengths):
        if n <= 0:
            assert not got[i].any()
            continue
        turned = rotate64(host64(q[i:i + 1]), [n - 1], 10000.0)[0]
        k, v = (P.rows(w, i, n) for w in (0, 1))
        for h in range(hq):
            o, tol = attend_shared(turned[h:h + 1], k[:, h // per], v[:, h // per], softmax_scale or 1 / math.sqrt(d))
            assert (np.abs(got[i, h] - o[0]) <= tol[0]).all(), (i, h)


# ------------------------------------------------------------------------------------------
# More prompts than one call takes
# ------------------------------------------------------------------------------------------
def _one_page_each(k, hq, hkv, d, page, sharing, seed):
    """k prompts of up to `page` rows in a page of their own, behind a page that each `sharing` of them have in common."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    firsts = -(-k // sharing)
    at = torch.arange(k, device="cuda", dtype=torch.int32)
    table = torch.stack([at // sharing, firsts + at], 1).contiguous()
    pools = [torch.randn((firsts + k, hkv, page, d), device="cuda", dtype=BF16, generator=g) for _ in range(2)]
    lengths = torch.randint(page, 2 * page, (k,), dtype=torch.int32, device="cuda", generator=g)
    lengths[::97] = -1
    new = torch.randn((k, hq + 2 * hkv, d), device="cuda", dtype=BF16, generator=g)          # (as a fused projection leaves them)
    return PagedCaches(*pools, table), lengths, new[:, :hq], new[:, hq:hq + hkv], new[:, hq + hkv:]


def _check_every_prompt(caches, n_rows, q, out, shared):
    """O of every prompt (n_rows that it attends to, < 0: none, O is 0) against the float64 form, over the pages as they are."""
    k, hq, d = q.shape
    page, active = caches.page_size, n_rows >= 0
    assert bool((out[~active] == 0).all())
    n = n_rows.clamp(min=1)
    rows = [x[caches.page_table.long()].movedim(2, 1).reshape(k, caches.hkv, -1, d).double() for x in (caches.k_pages, caches.v_pages)]
    theta = 10000.0 ** (-torch.arange(d // 2, device="cuda", dtype=torch.float64) / (d // 2))
    angle = ((n - 1).double()[:, None] * theta)[:, None]
    a, b = q.double()[..., :d // 2], q.double()[..., d // 2:]
    turned = torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1).view(k, caches.hkv, -1, d)
    s = torch.einsum("kgmd,kgrd->kgmr", turned, rows[0]) / math.sqrt(d)
    s = s.masked_fill(torch.arange(s.shape[-1], device="cuda") >= n[:, None, None, None], -math.inf)
    p = torch.softmax(s, -1)
    want = torch.einsum("kgmr,kgrd->kgmd", p, rows[1])
    # O is rounded to bf16 once: 2^-8 of it. A query reaches the products as two bf16 numbers (2^-16 of it), 2^-17 for the rotation and a sum
    # of 64 products in fp32: that moves a score by at most e = (that) sum |q k| scale, and so a weight over the sum of them by a factor of
    # exp(2 e) at most. A weight is one bf16 number over shared rows (2^-8 of it), else two (2^-15); 2^-17 for the sums over a few dozen
    # rows in fp32. All of it times sum p |v|.
    part = 2.0 ** -8 if shared else 2.0 ** -15
    e = torch.einsum("kgmd,kgrd->kgmr", turned.abs(), rows[0].abs()).amax(-1, keepdim=True) / math.sqrt(d) * (2.0 ** -16 + 2.0 ** -17)
    err = torch.einsum("kgmr,kgrd->kgmd", p, rows[1].abs()) * (torch.exp(2 * e) - 1 + part + 2.0 ** -17) * (1 + part)
    tol = want.abs() * 2.0 ** -8 + err * (1 + 2.0 ** -8)
    off = ((out.double().view_as(want) - want).abs() <= tol).flatten(1).all(1) | ~active
    assert bool(off.all()), (~off).nonzero()[:8]


@pytest.mark.gpu
@pytest.mark.parametrize("fresh", [True, False])
@pytest.mark.parametrize("k,sharing", [(16384, 0), (16384, 256), (8193, 300), (20000, 6000), (8192, 64)])
def test_step_of_more_prompts_than_a_call_takes(k, sharing, fresh):
    """Up to 64 groups of 256 samples, groups that lie on both sides of a cut, rows of no prompt: O of every prompt, and the pages are those
    that an append of the same rows leaves."""
    hq, hkv, d, page = 2, 1, 64, 16
    caches, lengths, q, kn, vn = _one_page_each(k, hq, hkv, d, page, sharing or 1, seed=k + sharing)
    pools = caches.k_pages.clone(), caches.v_pages.clone()
    groups = None
    if sharing:
        starts = list(range(0, k, sharing)) + [k]
        groups = tuple(torch.tensor(x, dtype=torch.int32, device="cuda") for x in (starts, [page] * (len(starts) - 1)))
    dec = PagedDecoder(caches, hq, 10000.0)
    out = dec.step(lengths, q, *((kn, vn) if fresh else (None, None)), groups=groups)
    assert dec.device_status() == 0
    _check_every_prompt(caches, lengths + fresh * (lengths >= 0).int(), q, out, bool(sharing))
    if fresh:
        again = PagedCaches(*pools, caches.page_table)
        prompt = torch.arange(k, dtype=torch.int32, device="cuda")
        again.append(torch.where(lengths >= 0, prompt, torch.full_like(prompt, -1)), lengths, kn, vn, 10000.0)
    assert torch.equal(caches.k_pages, pools[0]) and torch.equal(caches.v_pages, pools[1])


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [[0, 9000, 100, 16384], [0, 6000, 5000, 16384], [-1, 100, 200, 300], [0, 1, 2, 16385]])
def test_bad_groups_of_more_prompts_than_a_call_takes(bad):
    """Said to be bad for all of the prompts, whichever part of them a call is made for: nothing is shared."""
    hq, hkv, d, page, k = 2, 1, 64, 16, 16384
    caches, lengths, q, _, _ = _one_page_each(k, hq, hkv, d, page, 1, seed=9)
    groups = torch.tensor(bad, dtype=torch.int32, device="cuda"), torch.full((3,), page, dtype=torch.int32, device="cuda")
    dec = PagedDecoder(caches, hq, 10000.0)
    out = dec.step(lengths, q, groups=groups)
    assert dec.device_status() == pp.PP_PAGED_BAD_GROUPS
    _check_every_prompt(caches, lengths, q, out, False)


def test_more_groups_than_prompts_of_a_call_are_refused():
    caches = PagedCaches(*(torch.zeros(1, 1, 16, 64, dtype=BF16) for _ in range(2)), torch.zeros(9000, 1, dtype=torch.int32))
    ints = lambda n: torch.zeros(n, dtype=torch.int32)
    with pytest.raises(ValueError, match="groups"):
        PagedDecoder(caches, 1, 10000.0).step(ints(9000), torch.zeros(9000, 1, 64, dtype=BF16), groups=(ints(4502), ints(4501)))


# ------------------------------------------------------------------------------------------
# From the prefill into pages
# ------------------------------------------------------------------------------------------
def _prefill(lengths, hkv, d):
    """What `append_prefill` looks at before it makes a call."""
    return SimpleNamespace(hkv=hkv, d=d, k=len(lengths), lengths=np.array(lengths, np.int32))


def test_a_prefill_that_does_not_fit_is_refused():
    caches = PagedCaches.allocate(3, 20, 100, 8, 64, page_size=16, device="cpu")
    for i, rows in enumerate((40, 100, 0)):
        caches.reserve(i, rows)
    table = PagedCaches(caches.k_pages, caches.v_pages, caches.page_table)     # (the table is the caller's: up to its rows' ends)
    for c, lengths, hkv, d, start, says in [
        (caches, [5, 5], 4, 128, 0, "heads"), (caches, [5, 5], 8, 128, 0, "heads"), (caches, [5, 5], 4, 64, 0, "heads"),
        (caches, [1, 1, 0, 0], 8, 64, 0, "4 prompts"), (caches, [49, 100], 8, 64, 0, "prompt 0"), (caches, [48, 100, 1], 8, 64, 0, "prompt 2"),
        (table, [5, 113], 8, 64, 0, "prompt 1"), (caches, [5, 5], 8, 64, 6, "start"), (caches, [5, 5], 8, 64, [0, -1], "start"),
        (caches, [5, 5], 8, 64, [0, 0, 0], "shape"),
    ]:
        with pytest.raises(ValueError, match=says):
            c.append_prefill(_prefill(lengths, hkv, d), start)


@pytest.mark.gpu
@pytest.mark.parametrize("mode", ["packed", "padded"])
def test_a_prefill_leaves_rows_before_its_start(mode):
    """Prompts behind a prefix: the first one's pages are shared, and the others' prefill leaves them as they are. In all of them stand the
    bits that an append of every row leaves."""
    lengths, hq, hkv, d, page = np.array([70, 33, 48, 90], np.int32), 4, 2, 64, 16
    pre = PrefillBatch(lengths, hq, hkv, d, 10000.0, mode=mode)
    pre.load(*(normal((int(lengths.sum()), h, d), s) for s, h in enumerate((hq, hkv, hkv))))
    pre.run_fused()
    whole, behind = (PagedCaches.allocate(4, 30, 100, hkv, d, page) for _ in range(2))
    for i, n in enumerate(lengths):
        whole.reserve(i, int(n))
    assert torch.equal(whole.append_prefill(pre).cpu(), torch.from_numpy(lengths))
    behind.reserve(0, 70)
    start = [0]
    for i in range(1, 4):
        start.append(behind.share(0, i, 40))
        behind.reserve(i, int(lengths[i]))
    assert start == [0, 32, 32, 32]
    shared = behind.page_table[0, :2].long()
    for pool in (behind.k_pages, behind.v_pages):
        pool[shared] = 7
    behind.append_prefill(pre, [32, 32, 32, 32])
    assert all(bool((pool[shared] == 7).all()) for pool in (behind.k_pages, behind.v_pages))
    behind.append_prefill(pre, np.array(start))
    assert int(whole.status) == int(behind.status) == 0
    for a, b in ((whole.k_pages, behind.k_pages), (whole.v_pages, behind.v_pages)):
        for i, n in enumerate(int(x) for x in lengths):
            first = 0 if i == 0 else 2
            rows = lambda pool, c: pool[c.page_table[i, first:-(-n // page)].long()].transpose(1, 2).reshape(-1, hkv, d)[:n - first * page]
            assert torch.equal(rows(a, whole), rows(b, behind)) and bool(rows(a, whole).any() or i == 1)
        assert torch.equal(a[whole.page_table[0, :2].long()], b[shared])


# ------------------------------------------------------------------------------------------
# Kernels one behind the other
# ------------------------------------------------------------------------------------------
def test_no_kernel_lets_the_next_one_start_before_its_own_wait():
    """What the step reads ahead of its wait (lengths, table, rows that were there) is complete only because of that."""
    seen = 0
    for name in ("pp_paged.cu", "pp_paged_shared.cu"):
        with open(os.path.join(os.path.dirname(pp.__file__), "csrc", name)) as f:
            lines = [line.split("//")[0].strip() for line in f]
        for at, line in enumerate(lines):
            if line == "pdl_launch_dependents();":
                seen += 1
                assert lines[at - 1] == "pdl_wait();", (name, at + 1)
    assert seen == 6


# ------------------------------------------------------------------------------------------
# Status words
# ------------------------------------------------------------------------------------------
def test_status_words_are_read_and_reset():
    caches = PagedCaches.allocate(2, 4, 32, 1, 64, page_size=16, device="cpu")
    for x in (caches, PagedDecoder(caches, 1, 10000.0)):
        assert x.device_status() == 0
        x.status.fill_(pp.PP_PAGED_BAD_PAGE)
        assert x.device_status() == pp.PP_PAGED_BAD_PAGE == x.device_status()
        x.reset_status()
        assert x.device_status() == 0


@pytest.mark.gpu
def test_a_reset_status_word_tells_of_the_next_mistake():
    caches = PagedCaches.allocate(2, 4, 32, 1, 64, page_size=16)
    caches.reserve(0, 32)
    _, k, v = new_rows(1, 1, 1, 64, 3, False)
    one = lambda x: torch.tensor([x], dtype=torch.int32, device="cuda")
    dec = PagedDecoder(caches, 1, 10000.0)
    for prompt, position, code in ((5, 0, pp.PP_PAGED_BAD_PROMPT), (0, 32, pp.PP_PAGED_BAD_POSITION), (0, 31, 0), (1, 0, pp.PP_PAGED_BAD_PAGE)):
        caches.append(one(prompt), one(position), k, v, 10000.0)
        assert caches.device_status() == code
        caches.append(one(7), one(0), k, v, 10000.0)
        assert caches.device_status() == (code or pp.PP_PAGED_BAD_PROMPT)            # the first one stays
        caches.reset_status()
    q = new_rows(2, 1, 1, 64, 4, False)[0]
    for lengths, code in (([40, -1], pp.PP_PAGED_BAD_LENGTH), ([32, -1], 0), ([5, 5], pp.PP_PAGED_BAD_PAGE)):
        dec.step(torch.tensor(lengths, dtype=torch.int32, device="cuda"), q)
        assert dec.device_status() == code
        dec.reset_status()


# ------------------------------------------------------------------------------------------
# Captured steps, layers
# ------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("prompts,sharing,hq,hkv,d", [(3, 3, 8, 1, 128), (40, 40, 8, 1, 128), (16, 8, 4, 4, 64), (9000, 300, 2, 1, 64), (9000, 0, 2, 1, 64)])
def test_captured_step_is_the_step(prompts, sharing, hq, hkv, d):
    """With few and many queries of a group, and of more prompts than one call takes: replays over new queries and lengths."""
    caches, lengths, q, kn, vn = _one_page_each(prompts, hq, hkv, d, 16, sharing or 1, seed=prompts)
    starts = list(range(0, prompts, sharing or prompts)) + [prompts]
    groups = tuple(torch.tensor(x, dtype=torch.int32, device="cuda") for x in (starts, [16] * (len(starts) - 1))) if sharing else None
    dec, eager = PagedDecoder(caches, hq, 10000.0), PagedDecoder(caches, hq, 10000.0)
    out, g = torch.zeros_like(q, memory_format=torch.contiguous_format), torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        dec.step(lengths, q, kn, vn, out=out, groups=groups)
    stream.synchronize()
    with torch.cuda.graph(g, stream=stream):
        dec.step(lengths, q, kn, vn, out=out, groups=groups)
    for turn in range(3):
        lengths.copy_(torch.where(lengths < 0, lengths, 16 + (lengths + 5 * turn) % 16))
        for x in (q, kn, vn):
            x.copy_(x.roll(turn + 1, 0).clone())
        out.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            g.replay()
        stream.synchronize()
        assert torch.equal(out, eager.step(lengths, q, kn, vn, groups=groups)) and bool(out.any())
    assert dec.device_status() == eager.device_status() == 0


def test_layers_share_a_table():
    first = PagedCaches.allocate(2, 8, 60, 2, 64, page_size=16, device="cpu")
    second = PagedCaches(torch.zeros_like(first.k_pages), torch.zeros_like(first.v_pages), first.page_table)
    first.reserve(0, 40)
    assert second.page_table is first.page_table and second.struct.page_table == first.struct.page_table
    with pytest.raises(ValueError):
        second.reserve(1, 16)                          # (pages are handed out in one place)
