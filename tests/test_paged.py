"""The paged cache: rows appended to pages (pp_paged_append), the generation step over them (pp_paged_decode_step) and that step
for prompts that share pages (pp_paged_decode_shared), against plain float64 forms of their formulas."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2404_09529_b200 as pp
from paper_2404_09529_b200.runner import DecodeBatch, PagedCaches, PagedDecoder, PrefillBatch
from parity_utils import MAX_ABS_TOL, MEAN_ABS_TOL

E4M3 = torch.float8_e4m3fn
BF16 = torch.bfloat16


# ------------------------------------------------------------------------------------------
# Plain forms, float64 on the host
# ------------------------------------------------------------------------------------------
def host64(x):
    return x.detach().to("cpu").to(torch.float32).numpy().astype(np.float64)


def rotate64(x, position, base):
    """x [n, heads, d] rotated by its row's position."""
    half = x.shape[-1] // 2
    angle = np.asarray(position, np.float64)[:, None] * float(base) ** (-np.arange(half) / half)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


class Pages:
    """Two pools with random contents, a shuffled table and what they stand for. Every row that no prompt has is NaN, and so are
    the table's entries past a prompt's pages -1."""

    def __init__(self, room, hkv, d, page, rows_first, dtype, seed, common=None, spare=3, scale=1.0):
        g = np.random.default_rng(seed)
        room = np.asarray(room, np.int64)
        count = -(-room // page)
        common = np.zeros(len(room), np.int64) if common is None else common         # per prompt: (source prompt, pages)
        self.page, self.hkv, self.d, self.dtype, self.rows_first = page, hkv, d, dtype, rows_first
        own = [int(c) for c in count]
        for i, src in enumerate(common):
            if isinstance(src, tuple):
                own[i] = int(count[i]) - src[1]
        n_pages = sum(own) + spare
        ids = g.permutation(n_pages).astype(np.int32)
        table = np.full((len(room), max(int(count.max()), 1) + 1), -1, np.int32)
        at = 0
        for i in range(len(room)):
            skip = 0
            if isinstance(common[i], tuple):
                src, skip = common[i]
                table[i, :skip] = table[src, :skip]
            table[i, skip:count[i]] = ids[at:at + own[i]]
            at += own[i]
        self.table = table
        shape = (n_pages, page, hkv, d) if rows_first else (n_pages, hkv, page, d)
        self.k_scale = self.v_scale = None
        pools = [torch.from_numpy(scale * g.standard_normal(shape)).to(BF16) for _ in range(2)]
        if dtype == E4M3:
            self.k_scale, self.v_scale = (torch.from_numpy(0.014 + 0.031 * g.random(hkv)).float() for _ in range(2))
            pools = [(p.float() / s.view((-1, 1) if rows_first else (-1, 1, 1))).to(E4M3) for p, s in zip(pools, (self.k_scale, self.v_scale))]
        self.pools = pools

    def poison(self, lengths):
        """NaN in every row that is not below its prompt's length."""
        kept = {(int(self.table[i, p // self.page]), p % self.page) for i, n in enumerate(lengths) for p in range(max(int(n), 0))}
        n_pages = self.pools[0].shape[0]
        for page in range(n_pages):
            for row in range(self.page):
                if (page, row) not in kept:
                    for p in self.pools:
                        p.view(torch.uint8 if self.dtype == E4M3 else torch.int16)[(page, row) if self.rows_first else (page, slice(None), row)] = 0x7F if self.dtype == E4M3 else 0x7FC0

    def cuda(self):
        to = lambda x: None if x is None else x.cuda()
        self.caches = PagedCaches(self.pools[0].cuda(), self.pools[1].cuda(), torch.from_numpy(self.table).cuda(), self.rows_first,
                                  to(self.k_scale), to(self.v_scale))
        return self.caches

    def rows(self, which, i, n, pools=None):
        """Rows 0 .. n - 1 of prompt i, [n, hkv, d] float64."""
        pool = (pools or self.pools)[which]
        pos = np.arange(n)
        page, row = torch.from_numpy(self.table[i, pos // self.page].astype(np.int64)), torch.from_numpy(pos % self.page)
        cells = pool.view(torch.uint8)[(page, row) if self.rows_first else (page, slice(None), row)].view(self.dtype) if self.dtype == E4M3 \
            else pool[(page, row) if self.rows_first else (page, slice(None), row)]
        x = host64(cells)
        scale = (self.k_scale, self.v_scale)[which]
        return x if scale is None else x * host64(scale)[:, None]


def stored64(x, dtype, scale):
    """x [.., hkv, d] float64 as the pages hold it."""
    if dtype == BF16:
        return host64(torch.from_numpy(x).to(torch.float32).to(BF16))
    s = host64(scale)[:, None]
    return host64(torch.from_numpy(np.clip(x / s, -448, 448)).to(torch.float32).to(E4M3)) * s


def attend64(q, keys, values, scale):
    """q [hq, d], keys and values [n, hkv, d] -> O [hq, d] and, of every query head, the largest sum of |q_d k_d| and |v|."""
    hq, d = q.shape
    hkv = keys.shape[1]
    o, size, big = np.zeros((hq, d)), np.zeros(hq), np.zeros(hq)
    for h in range(hq if len(keys) else 0):
        kv = h // (hq // hkv)
        s = keys[:, kv] @ q[h] * scale
        p = np.exp(s - s.max())
        o[h] = (p / p.sum()) @ values[:, kv]
        size[h] = (np.abs(keys[:, kv]) @ np.abs(q[h])).max() * scale
        big[h] = np.abs(values[:, kv]).max()
    return o, size, big


def step_bound(o, size, big, n, d, dtype=BF16):
    """How far a step's O may be off. A query reaches the products in two 16-bit parts (2^-16 of it is lost; over 8-bit pages it is
    rounded to f16 once, and so are the weights: 2^-12, and 2^-35 for those that f16 has no bits for) after a rotation in
    fp32 (3 roundings), a score is a sum of 2 d products in fp32 (2 d 2^-24 of the sum of magnitudes, twice that for
    tensor cores that truncate), its exponential has 2^-22, and a weight too reaches the products in two 16-bit parts (2^-16): a score
    or the logarithm of a weight that is off by e moves O by at most 2 e max|v|. Sums of n
    weights and products in fp32: n 2^-23 max|v|. The last rounding: 2^-8 of O (half of a step of bf16)."""
    part = 2.0 ** -16 if dtype == BF16 else 2.0 ** -12
    e = size * (part + (4 * d + 8) * 2.0 ** -24) + part + 2.0 ** -22
    lost = n * 2.0 ** -23 if dtype == BF16 else n * (2.0 ** -23 + 2.0 ** -35)
    return np.abs(o) * 2.0 ** -8 + ((2 * e + lost + 64 * 2.0 ** -23) * big)[:, None] + 1e-30


def normal(shape, seed):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape)).to(BF16)


def new_rows(n, hq, hkv, d, seed, fused):
    """q, k, v of n rows on the device: tensors of their own or slices of one."""
    whole = normal((n, hq + 2 * hkv, d), seed).cuda()
    parts = whole[:, :hq], whole[:, hq:hq + hkv], whole[:, hq + hkv:]
    return parts if fused else tuple(x.contiguous() for x in parts)


def check_step(P, lengths, q, k, v, got, before, base, softmax_scale=0.0, loose=None):
    """O of every prompt, and the pages: the new row, and nothing else, has changed. before: the pools before the step."""
    caches = P.caches
    after = [x.cpu() for x in (caches.k_pages, caches.v_pages)]
    want = [x.clone() for x in before]
    fresh = k is not None
    scale = softmax_scale or 1 / math.sqrt(P.d)
    errors = []
    for i, n in enumerate(int(x) for x in lengths):
        if n < 0:
            continue
        position = n if fresh else max(n - 1, 0)
        keys, values = P.rows(0, i, n, before), P.rows(1, i, n, before)
        if fresh:
            k_row = rotate64(host64(k[i:i + 1]), [n], base)
            v_row = host64(v[i:i + 1])
            page, row = int(P.table[i, n // P.page]), n % P.page
            cell = (page, row) if P.rows_first else (page, slice(None), row)
            for which, (exact, source) in enumerate(((k_row, k), (v_row, v))):
                bytes_ = lambda x: x.view(torch.uint8 if P.dtype == E4M3 else torch.int16)
                stored = P.rows(which, i, n + 1, after)[n]
                check_stored(stored, exact[0], P.dtype, (P.k_scale, P.v_scale)[which], host64(source[i]), copied=which == 1)
                bytes_(want[which])[cell] = bytes_(after[which])[cell]
            keys = np.concatenate([keys, P.rows(0, i, n + 1, after)[n:]])
            values = np.concatenate([values, P.rows(1, i, n + 1, after)[n:]])
        o, size, big = attend64(rotate64(host64(q[i:i + 1]), [position], base)[0], keys, values, scale)
        err = np.abs(host64(got[i]) - o)
        assert np.isfinite(host64(got[i])).all(), i
        if loose is None:
            assert (err <= step_bound(o, size, big, len(keys), P.d, P.dtype)).all(), (i, n, err.max())
        errors.append(err.ravel())
    if loose is not None and errors:
        e = np.concatenate(errors)
        assert e.max() <= loose[0] and e.mean() <= loose[1], (e.max(), e.mean())
    for w, a in zip(want, after):
        raw = torch.uint8 if P.dtype == E4M3 else torch.int16
        assert torch.equal(w.view(raw), a.view(raw)), "pages beside the new rows were written"


def check_stored(stored, exact, dtype, scale, source, copied):
    """A stored row against its exact value: half of a step of its type, and for a key the rotation in fp32 (2^-22 of the magnitudes)."""
    if dtype == BF16:
        if copied:
            assert np.array_equal(stored, source)
            return
        bound = np.abs(exact) * 2.0 ** -8
    else:
        s = host64(scale)[:, None]
        exact = np.clip(exact, -448 * s, 448 * s)
        bound = np.maximum(np.abs(exact) * 2.0 ** -4, 2.0 ** -10 * s) * (1 + 2.0 ** -20)
    half = exact.shape[-1] // 2
    magnitude = np.tile(np.abs(source[..., :half]) + np.abs(source[..., half:]), 2)
    assert (np.abs(stored - exact) <= bound + magnitude * 2.0 ** -22).all()


# ------------------------------------------------------------------------------------------
# Host: arguments and the pages' bookkeeping
# ------------------------------------------------------------------------------------------
def _cache(**changes):
    c = pp.PagedCache(0x1000, 0x1000, None, None, 0x1000, 4 * 16 * 64, 16 * 64, 64, 8, 16, 4, pp.PP_CACHE_BF16)
    for name, value in changes.items():
        setattr(c, name, value)
    return c


def _params(hq=8, hkv=4, d=64, base=10000.0, scale=0.0, flags=0):
    return pp.AttnParams(hq, hkv, d, base, scale, 1, 1, flags)


INVALID, SMALL, UNSUPPORTED, ALIGNMENT, TOO_LARGE = -1, -3, -4, -5, -9

CACHE_REFUSALS = [
    (dict(k_pages=None), INVALID), (dict(v_pages=None), INVALID), (dict(page_table=None), INVALID), (dict(n_pages=0), INVALID),
    (dict(table_stride=0), INVALID), (dict(page_stride=0), INVALID), (dict(head_stride=-64), INVALID), (dict(row_stride=32), INVALID),
    (dict(type=2), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(page_size=512), UNSUPPORTED),
    (dict(table_stride=1 << 27), UNSUPPORTED), (dict(row_stride=68), ALIGNMENT), (dict(k_pages=0x1008), ALIGNMENT),
    (dict(v_pages=0x1002), ALIGNMENT), (dict(page_table=0x1002), ALIGNMENT), (dict(type=pp.PP_CACHE_E4M3), INVALID),
    (dict(type=pp.PP_CACHE_E4M3, k_scale=0x1000, v_scale=0x1000, row_stride=72), ALIGNMENT),
]


def _append(params=None, cache=None, prompt=0x1000, position=0x1000, n_rows=3, n_prompts=2, k=0x1000, k_stride=0, v=0x1000, v_stride=0):
    pp.pp_paged_append(params or _params(), cache or _cache(), prompt, position, n_rows, n_prompts, k, k_stride, v, v_stride)


def _step(params=None, cache=None, lengths=0x1000, k=2, q=0x1000, q_stride=0, k_new=0x1000, k_stride=0, v_new=0x1000, v_stride=0, o=0x1000,
          ws=0x1000, ws_bytes=1 << 40, groups=None):
    params, cache = params or _params(), cache or _cache()
    if groups is None:
        pp.pp_paged_decode_step(params, cache, lengths, k, q, q_stride, k_new, k_stride, v_new, v_stride, o, ws, ws_bytes)
    else:
        pp.pp_paged_decode_shared(params, cache, lengths, k, *groups, q, q_stride, k_new, k_stride, v_new, v_stride, o, ws, ws_bytes)


def _refused(status, call, *args, **kwargs):
    with pytest.raises(pp.PrepackError) as err:
        call(*args, **kwargs)
    assert err.value.status == status, (err.value, args, kwargs)


def test_append_refusals():
    for changes, status in CACHE_REFUSALS:
        _refused(status, _append, cache=_cache(**changes))
    for kwargs, status in [
        (dict(params=_params(d=96)), UNSUPPORTED), (dict(params=_params(base=0.0)), INVALID), (dict(params=_params(hkv=0)), INVALID),
        (dict(params=_params(flags=2)), INVALID), (dict(params=_params(flags=8)), INVALID), (dict(n_rows=-1), INVALID),
        (dict(n_prompts=0), INVALID), (dict(prompt=None), INVALID), (dict(position=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID),
        (dict(k_stride=255), INVALID), (dict(v_stride=-256), INVALID), (dict(k_stride=260), ALIGNMENT), (dict(k=0x1004), ALIGNMENT),
        (dict(prompt=0x1001), ALIGNMENT),
    ]:
        _refused(status, _append, **kwargs)
    _append(n_rows=0)                                  # nothing to do, nothing launched
    _append(n_rows=0, prompt=None, position=None, k=None, v=None)


def test_step_refusals():
    for changes, status in CACHE_REFUSALS:
        _refused(status, _step, cache=_cache(**changes))
        _refused(status, _step, cache=_cache(**changes), groups=(0x1000, 0x1000, 1))
    for kwargs, status in [
        (dict(params=_params(d=32)), UNSUPPORTED), (dict(params=_params(hq=6)), UNSUPPORTED), (dict(params=_params(hq=36)), UNSUPPORTED),
        (dict(params=_params(hq=0)), INVALID), (dict(params=_params(base=-1.0)), INVALID), (dict(params=_params(scale=-1.0)), INVALID),
        (dict(params=_params(scale=math.nan)), INVALID), (dict(params=_params(flags=1)), INVALID), (dict(lengths=None), INVALID), (dict(k=0), INVALID),
        (dict(q=None), INVALID), (dict(o=None), INVALID), (dict(ws=None), INVALID), (dict(k_new=None), INVALID), (dict(v_new=None), INVALID),
        (dict(q_stride=8 * 64 - 8), INVALID), (dict(k_stride=4 * 64 + 4), ALIGNMENT), (dict(v_stride=8), INVALID),
        (dict(k=8193), TOO_LARGE), (dict(ws=0x1080), ALIGNMENT), (dict(q=0x1008), ALIGNMENT), (dict(o=0x1002), ALIGNMENT), (dict(lengths=0x1002), ALIGNMENT),
        (dict(ws_bytes=16), SMALL),
    ]:
        _refused(status, _step, **kwargs)
        _refused(status, _step, **kwargs, groups=(0x1000, 0x1000, 1) if kwargs.get("k", 2) else (0x1000, 0x1000, 1))
    for groups, status in [((None, 0x1000, 1), INVALID), ((0x1000, None, 1), INVALID), ((0x1000, 0x1000, 0), INVALID), ((0x1000, 0x1000, -1), INVALID),
                           ((0x1000, 0x1000, 3), INVALID), ((0x1002, 0x1000, 1), ALIGNMENT)]:
        _refused(status, _step, groups=groups)
    _refused(UNSUPPORTED, _step, cache=_cache(type=pp.PP_CACHE_E4M3, k_scale=0x1000, v_scale=0x1000), groups=(0x1000, 0x1000, 1))


def test_workspace_bytes():
    ask = pp.pp_paged_decode_workspace_bytes
    p = _params()
    # parts of what is cut, whose number does not depend on k, and the prepared queries: a word an element, a factor a head
    assert 0 < ask(p, 1) and abs(ask(p, 8192) - ask(p, 1) - 8191 * p.n_q_heads * (p.head_dim + 1) * 4) < 512      # (each on a boundary of 256)
    assert ask(_params(), 4, 4) > ask(_params(), 4, 1) - 1 > ask(_params(), 4)
    assert [ask(_params(), k, g) for k, g in ((0, 0), (8193, 0), (4, 5), (4, -1))] == [0] * 4
    assert ask(_params(hq=6), 4) == 0 and ask(_params(d=80), 4) == 0
    # room for a step over a cache that is wide and long depends on neither
    small = _step
    _refused(SMALL, small, ws_bytes=ask(_params(), 2) - 1)
    _refused(SMALL, small, ws_bytes=ask(_params(), 2, 1) - 1, groups=(0x1000, 0x1000, 1))


def test_mirror_of_the_cache_structure():
    assert ctypes.sizeof(pp.PagedCache) == 5 * 8 + 3 * 8 + 4 * 4


def test_pages_are_handed_out_shared_and_given_back():
    c = PagedCaches.allocate(4, 10, 100, 2, 64, page_size=16, device="cpu")
    assert c.page_table.shape == (4, 7) and bool((c.page_table == -1).all())
    c.reserve(0, 33)
    assert (c.page_table[0] >= 0).sum() == 3
    before = c.page_table[0].clone()
    c.reserve(0, 48)                                   # they are there
    assert torch.equal(before, c.page_table[0])
    c.reserve(0, 49)
    assert torch.equal(before[:3], c.page_table[0][:3]) and (c.page_table[0] >= 0).sum() == 4
    assert c.share(0, 1, 40) == 32                     # whole pages
    assert torch.equal(c.page_table[1][:2], c.page_table[0][:2]) and int(c.page_table[1][2]) == -1
    c.reserve(1, 70)
    used = torch.cat([c.page_table[0][:4], c.page_table[1][2:5]])
    assert len(set(used.tolist())) == 7
    with pytest.raises(ValueError):
        c.share(0, 1, 16)                              # has pages already
    with pytest.raises(ValueError):
        c.share(2, 3, 16)                              # nothing to share
    with pytest.raises(ValueError):
        c.reserve(2, 113)                              # past the row of the table
    with pytest.raises(MemoryError):
        c.reserve(2, 64)                               # 3 of 10 pages are left
    assert int(c.page_table[2][0]) == -1
    c.release(0)                                       # the two shared pages stay with prompt 1
    assert bool((c.page_table[0] == -1).all())
    c.reserve(2, 80)
    assert not set(c.page_table[2][:5].tolist()) & set(c.page_table[1][:5].tolist())
    c.release(1)
    c.release(2)
    c.reserve(3, 112)
    assert len(set(c.page_table[3].tolist())) == 7


def test_caches_refuse_tensors_that_do_not_fit():
    k = torch.zeros(4, 2, 16, 64, dtype=BF16)
    table = torch.zeros(2, 3, dtype=torch.int32)
    PagedCaches(k, k.clone(), table)
    s = torch.ones(2)
    for args in [(k.float(), k.float(), table), (k, k[:3], table), (k, k.transpose(0, 1), table), (k, k, table.long()), (k, k, table.t()),
                 (k, k, table, False, s, s), (k.to(E4M3), k.to(E4M3), table), (k.to(E4M3), k.to(E4M3), table, False, s, s.double()),
                 (k.to(E4M3), k.to(E4M3), table, False, s, torch.ones(3)), (k[..., ::2], k[..., ::2], table)]:
        with pytest.raises(ValueError):
            PagedCaches(*args)
    c = PagedCaches(k, k.clone(), table)
    with pytest.raises(ValueError):
        c.reserve(0, 1)                                # the table is the caller's
    x = torch.zeros(5, 2, 64, dtype=BF16)
    assert c.check_new(x, 5, 2, "x") == 128 and c.check_new(torch.zeros(5, 7, 64, dtype=BF16)[:, 3:5], 5, 2, "x") == 7 * 64
    for bad in (x.float(), x[:4], x[:, :1].expand(5, 2, 64), x[:1].expand(5, 2, 64), torch.zeros(5, 64, 2, dtype=BF16).transpose(1, 2),
                torch.zeros(5, 4, 64, dtype=BF16)[:, ::2]):
        with pytest.raises(ValueError):
            c.check_new(bad, 5, 2, "x")


# ------------------------------------------------------------------------------------------
# GPU: appending
# ------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("hkv,d,page,rows_first,dtype,fused,rotated", [
    (1, 64, 16, False, BF16, False, False), (4, 128, 32, True, BF16, True, False), (8, 128, 64, False, E4M3, True, False),
    (3, 64, 128, True, E4M3, False, False), (32, 128, 256, False, BF16, False, False), (40, 128, 16, True, BF16, True, False),
    (5, 128, 16, False, E4M3, False, True), (8, 64, 64, True, BF16, False, True),
])
def test_append(hkv, d, page, rows_first, dtype, fused, rotated):
    """Rows in a shuffled order, of prompts that have rows already and of none, at positions from 0 to far ones."""
    rng = np.random.default_rng(hkv * d + page)
    start, new = np.array([0, 15, 16, 250, 7000, 3]), np.array([37, 1, 0, 20, 11, 130])
    P = Pages(start + new, hkv, d, page, rows_first, dtype, seed=1)
    caches = P.cuda()
    cells = [(i, p) for i in range(len(new)) for p in range(start[i], start[i] + new[i])] + [(-1, 5)] * 9
    rng.shuffle(cells)
    prompt, position = (np.array([c[x] for c in cells], np.int32) for x in (0, 1))
    _, k, v = new_rows(len(cells), 1, hkv, d, 2, fused)
    k[prompt < 0] = float("nan")
    before = [x.clone() for x in P.pools]
    caches.append(torch.from_numpy(prompt).cuda(), torch.from_numpy(position).cuda(), k, v, 500000.0, rotated=rotated)
    assert int(caches.status) == 0
    after = [x.cpu() for x in (caches.k_pages, caches.v_pages)]
    raw = torch.uint8 if dtype == E4M3 else torch.int16
    for which, source in enumerate((k, v)):
        src = host64(source)
        for r, (i, p) in enumerate(cells):
            if i < 0:
                continue
            exact = src[r] if which or rotated else rotate64(src[r:r + 1], [p], 500000.0)[0]
            check_stored(P.rows(which, i, p + 1, after)[p], exact, dtype, (P.k_scale, P.v_scale)[which], src[r], copied=bool(which) or rotated)
            cell = (int(P.table[i, p // page]), p % page) if rows_first else (int(P.table[i, p // page]), slice(None), p % page)
            before[which].view(raw)[cell] = after[which].view(raw)[cell]
        assert torch.equal(before[which].view(raw), after[which].view(raw))


@pytest.mark.gpu
@pytest.mark.parametrize("d,hq,hkv,page,rows_first", [(128, 8, 2, 16, False), (64, 4, 4, 64, True)])
def test_append_after_prefill_is_unpack(d, hq, hkv, page, rows_first):
    """The packed keys that a prefill has rotated, copied into pages, and the raw ones, rotated on the way, are the bits of the caches
    that the prefill fills itself."""
    lengths = np.array([70, 3, 129, 64, 1, 33], np.int32)
    q, k, v = (normal((int(lengths.sum()), h, d), s) for s, h in enumerate((hq, hkv, hkv)))
    pre = PrefillBatch(lengths, hq, hkv, d, 10000.0)
    pre.load(q, k, v)
    pre.run_fused()
    by_copy, by_rotation = (PagedCaches.allocate(len(lengths), 40, 160, hkv, d, page, rows_first=rows_first) for _ in range(2))
    for c in (by_copy, by_rotation):
        for i, n in enumerate(lengths):
            c.reserve(i, int(n))
    assert torch.equal(by_copy.append_prefill(pre).cpu(), torch.from_numpy(lengths))
    prompt = torch.from_numpy(np.repeat(np.arange(len(lengths)), lengths).astype(np.int32)).cuda()
    position = torch.from_numpy(np.concatenate([np.arange(n) for n in lengths]).astype(np.int32)).cuda()
    by_rotation.append(prompt, position, k.cuda(), v.cuda(), 10000.0)
    for c in (by_copy, by_rotation):
        assert int(c.status) == 0
        table = c.page_table.cpu()
        for i, n in enumerate(int(x) for x in lengths):
            for pool, want in zip((c.k_pages, c.v_pages), pre.caches(i)):
                ids = table[i, :-(-n // page)].long().cuda()
                got = pool[ids] if rows_first else pool[ids].transpose(1, 2)            # [pages, row, head, d]
                assert torch.equal(got.reshape(-1, hkv, d)[:n].transpose(0, 1), want[:, :n])


@pytest.mark.gpu
def test_append_says_what_it_skips():
    for prompt, position, entry, code in [(2, 0, None, pp.PP_PAGED_BAD_PROMPT), (0, -1, None, pp.PP_PAGED_BAD_POSITION),
                                          (0, 48, None, pp.PP_PAGED_BAD_POSITION), (1, 20, -1, pp.PP_PAGED_BAD_PAGE),
                                          (1, 20, 7, pp.PP_PAGED_BAD_PAGE), (-7, -9, None, 0)]:
        k = torch.zeros(7, 2, 16, 64, dtype=BF16, device="cuda")
        table = torch.tensor([[0, 1, 2], [3, 4, 5]], dtype=torch.int32, device="cuda")
        if entry is not None:
            table[1, 1] = entry
        c = PagedCaches(k, k.clone(), table)
        new = torch.ones(3, 2, 64, dtype=BF16, device="cuda")
        c.append(torch.tensor([0, prompt, 1], dtype=torch.int32, device="cuda"), torch.tensor([5, position, 0], dtype=torch.int32, device="cuda"),
                 new, new, 10000.0, rotated=True)
        assert int(c.status) == code, (prompt, position, entry)
        want = torch.zeros_like(k)
        want[0, :, 5] = 1
        want[3, :, 0] = 1
        assert torch.equal(c.k_pages, want) and torch.equal(c.v_pages, want)


@pytest.mark.gpu
def test_append_keeps_nan_and_clamps_in_8_bits():
    P = Pages([16], 2, 64, 16, False, E4M3, seed=3)
    c = P.cuda()
    k = torch.full((1, 2, 64), 1.0, dtype=BF16, device="cuda")
    k[0, 0, 3], k[0, 0, 4], k[0, 1, 5], k[0, 1, 6] = float("nan"), float("inf"), -float("inf"), 1e6
    c.append(*(torch.tensor([x], dtype=torch.int32, device="cuda") for x in (0, 9)), k, k, 10000.0, rotated=True)
    page = int(P.table[0, 0])
    for pool in (c.k_pages, c.v_pages):
        row = pool[page, :, 9].float().cpu()
        assert torch.isnan(row[0, 3]) and [float(row[0, 4]), float(row[1, 5]), float(row[1, 6])] == [448, -448, 448]
        assert int(torch.isnan(row).sum()) == 1


# ------------------------------------------------------------------------------------------
# GPU: the generation step
# ------------------------------------------------------------------------------------------
EDGES = [0, 1, 2, 15, 16, 17, 31, 33, 47, 48, 49, 63, 64, 65, 127, 128, 129, 191, 193, 255, 256, 257]


@pytest.mark.gpu
@pytest.mark.parametrize("fresh", [True, False])
@pytest.mark.parametrize("hq,hkv,d,page,rows_first,dtype,fused", [
    (4, 4, 128, 16, False, BF16, False), (8, 1, 128, 32, True, BF16, True), (6, 2, 64, 64, False, BF16, False), (16, 2, 64, 256, True, BF16, True),
    (4, 4, 128, 128, True, E4M3, True), (8, 1, 128, 16, False, E4M3, False), (6, 2, 64, 16, True, E4M3, False), (8, 8, 64, 64, False, E4M3, True),
])
def test_step(hq, hkv, d, page, rows_first, dtype, fused, fresh):
    """Every remainder of a step of 16 keys, a block of 64 and a page, prompts without rows, rows of no prompt, on pages whose other
    rows are NaN."""
    lengths = np.array(EDGES[:12] + [-1] + EDGES[12:] + [-5, 600], np.int32)
    P = Pages(np.maximum(lengths, -1) + fresh, hkv, d, page, rows_first, dtype, seed=d + hq)
    P.poison(lengths)
    caches = P.cuda()
    q, k, v = new_rows(len(lengths), hq, hkv, d, 5, fused)
    q[12], k[12], v[12] = float("nan"), float("nan"), float("nan")
    before = [x.clone() for x in P.pools]
    out = torch.full((len(lengths), hq, d), 7.0, dtype=BF16, device="cuda")
    dec = PagedDecoder(caches, hq, 10000.0)
    args = (k, v) if fresh else (None, None)
    dec.step(torch.from_numpy(lengths).cuda(), q, *args, out=out)
    assert dec.device_status() == 0
    idle = torch.from_numpy(lengths < 0).cuda()
    assert bool((out[idle] == 7).all())
    if not fresh:
        assert bool((out[0] == 0).all())               # attends to nothing
    check_step(P, lengths, q, *args, out, before, 10000.0)


@pytest.mark.gpu
@pytest.mark.parametrize("lengths,hq,hkv,d,page,dtype,scale", [
    ([70000], 8, 2, 128, 64, BF16, 0.0), ([30001, 5], 2, 2, 64, 16, E4M3, 0.0), ([9000, 1, 4000, 64], 4, 1, 128, 256, E4M3, 0.3),
    ([2049, 4096, 4097, 8191], 32, 32, 64, 32, BF16, 0.05), ([17] * 300, 8, 4, 64, 16, BF16, 0.0), (list(range(700)), 2, 1, 128, 16, BF16, 0.0),
    ([3] * 8192, 1, 1, 64, 16, BF16, 0.0),
])
def test_step_over_many_chunks_and_many_prompts(lengths, hq, hkv, d, page, dtype, scale):
    lengths = np.array(lengths, np.int32)
    P = Pages(lengths + 1, hkv, d, page, False, dtype, seed=3)
    caches = P.cuda()
    q, k, v = new_rows(len(lengths), hq, hkv, d, 6, False)
    before = [x.clone() for x in P.pools]
    dec = PagedDecoder(caches, hq, 500000.0, softmax_scale=scale)
    out = dec.step(torch.from_numpy(lengths).cuda(), q, k, v)
    assert dec.device_status() == 0
    some = lengths.copy()
    if len(lengths) > 400:                             # (the plain form of a part of them; the pages of all)
        keep = np.zeros(len(lengths), bool)
        keep[::97] = True
        after = [x.cpu() for x in (caches.k_pages, caches.v_pages)]
        for i in np.nonzero(~keep)[0]:
            n = int(lengths[i])
            for w in range(2):
                before[w][int(P.table[i, n // page]), :, n % page] = after[w][int(P.table[i, n // page]), :, n % page]
        some[~keep] = -1
    check_step(P, some, q, k, v, out, before, 500000.0, scale)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_step_beyond_32_bits(dtype):
    """Pages whose elements lie more than 2^32 into the pools, at page and head strides that leave gaps."""
    hkv, d, page = 2, 128, 16
    size = 1 if dtype == E4M3 else 2
    n_pages, head_stride = 72, page * d + 64
    page_stride = 1 << 26                              # 72 pages of 2^26 elements: 4.8e9
    raw = [torch.empty(n_pages * page_stride * size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    pools = [torch.as_strided(x.view(dtype), (n_pages, hkv, page, d), (page_stride, head_stride, d, 1)) for x in raw]
    lengths = np.array([50, 100], np.int32)
    P = Pages(lengths + 1, hkv, d, page, False, dtype, seed=8, spare=0)
    for pool, x in zip(pools, P.pools):
        for p in range(x.shape[0]):
            pool.view(torch.uint8 if size == 1 else torch.int16)[n_pages - 1 - p].copy_(x.view(torch.uint8 if size == 1 else torch.int16)[p])
    table = torch.from_numpy(np.where(P.table < 0, -1, n_pages - 1 - P.table).astype(np.int32)).cuda()
    to = lambda s: None if s is None else s.cuda()
    far = PagedCaches(*pools, table, False, to(P.k_scale), to(P.v_scale))
    near = P.cuda()
    q, k, v = new_rows(2, 4, hkv, d, 9, False)
    ln = torch.from_numpy(lengths).cuda()
    a, b = (PagedDecoder(c, 4, 10000.0) for c in (far, near))
    assert torch.equal(a.step(ln, q, k, v), b.step(ln, q, k, v)) and a.device_status() == 0
    row = torch.tensor([1], dtype=torch.int32, device="cuda")
    for c in (far, near):
        c.append(row, row * 7, k[:1], v[:1], 10000.0)
    if dtype == BF16:
        g = (torch.tensor([0, 2], dtype=torch.int32, device="cuda"), torch.tensor([0], dtype=torch.int32, device="cuda"))
        assert torch.equal(a.step(ln, q, groups=g), b.step(ln, q, groups=g))
        one = (torch.tensor([1, 2], dtype=torch.int32, device="cuda"), torch.tensor([96], dtype=torch.int32, device="cuda"))
        assert torch.equal(a.step(ln, q, groups=one), b.step(ln, q, groups=one)) and a.device_status() == 0
    assert torch.equal(a.step(ln + 1, q), b.step(ln + 1, q))


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 128), (8, 1, 128), (6, 2, 64)])
def test_step_with_infinite_and_huge_values(hq, hkv, d):
    """An infinity among the values that a prompt has makes that element of O infinite (with both signs, or a NaN, not a number)
    and no other; the largest numbers of no weight add nothing; keys whose score is -inf weigh nothing."""
    lengths = np.array([1, 16, 17, 50, 64, 65, 200, 700], np.int32)
    P = Pages(lengths, hkv, d, 16, False, BF16, seed=hq + d)
    q = new_rows(len(lengths), hq, hkv, d, 11, False)[0]
    inf = float("inf")
    cell = lambda i, p: (int(P.table[i, p // 16]), slice(None), p % 16)
    for i, n in enumerate(int(x) for x in lengths):
        vals = P.pools[1]
        vals[cell(i, 0)][0, 1] = inf
        vals[cell(i, n - 1)][hkv - 1, d - 1] = -inf
        vals[cell(i, n // 2)][0, d // 2 + 3] = inf
        vals[cell(i, n - 1)][0, 8] = float("nan")
        vals[cell(i, n // 3)][0, 6] = inf
        vals[cell(i, n - 1)][0, 6] = -inf if n > 1 else inf
    P.poison(lengths)
    caches = P.cuda()
    got = PagedDecoder(caches, hq, 10000.0).step(torch.from_numpy(lengths).cuda(), q)
    for i, n in enumerate(int(x) for x in lengths):
        with np.errstate(invalid="ignore"):
            ref, size, _ = attend64(rotate64(host64(q[i:i + 1]), [n - 1], 10000.0)[0], P.rows(0, i, n), P.rows(1, i, n), 1 / math.sqrt(d))
        g = host64(got[i])
        assert np.isinf(ref).any() and np.isnan(ref).any()
        assert np.array_equal(np.isnan(g), np.isnan(ref)) and np.array_equal(g[np.isinf(ref)], ref[np.isinf(ref)]), i
        fine = np.isfinite(ref)
        big = np.full(hq, np.abs(P.rows(1, i, n)[np.isfinite(P.rows(1, i, n))]).max())
        assert (np.abs(g - np.where(fine, ref, 0))[fine] <= step_bound(np.where(fine, ref, 0), size, big, n, d)[fine]).all(), i


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_step_with_large_and_small_queries(dtype):
    """Queries of 1e-6 to 1e6 (with a softmax scale that brings the scores back): nothing overflows or is lost on the way to 16 bits."""
    lengths = np.array([40, 200, 90], np.int32)
    P = Pages(lengths, 2, 128, 16, False, dtype, seed=4)
    caches = P.cuda()
    for size in (1e-6, 1e-3, 1e3, 1e6):
        q = (new_rows(3, 4, 2, 128, 12, False)[0].float() * size).to(BF16)
        scale = 0.09 / size
        out = PagedDecoder(caches, 4, 10000.0, softmax_scale=scale).step(torch.from_numpy(lengths).cuda(), q)
        check_step(P, lengths, q, None, None, out, P.pools, 10000.0, scale)


@pytest.mark.gpu
def test_step_says_what_is_wrong():
    def run(lengths, table=None, fresh=True):
        P = Pages([40, 40], 2, 64, 16, False, BF16, seed=2)
        c = P.cuda()
        if table is not None:
            c.page_table[table[0], table[1]] = table[2]
        q, k, v = new_rows(2, 2, 2, 64, 3, False)
        before = c.k_pages.clone()
        dec = PagedDecoder(c, 2, 10000.0)
        out = torch.full((2, 2, 64), 7.0, dtype=BF16, device="cuda")
        dec.step(torch.tensor(lengths, dtype=torch.int32, device="cuda"), q, *((k, v) if fresh else (None, None)), out=out)
        return dec.device_status(), out, before, c
    room = 4 * 16
    status, out, before, c = run([30, room])           # no room for one more
    assert status == pp.PP_PAGED_BAD_LENGTH and bool((out[1] == 7).all()) and not bool((out[0] == 7).any())
    assert run([30, room + 1], fresh=False)[0] == pp.PP_PAGED_BAD_LENGTH
    assert run([30, 2 ** 31 - 1])[0] == pp.PP_PAGED_BAD_LENGTH
    for entry in (-1, 1000, 2 ** 31 - 1, -2 ** 31):
        status, out, before, c = run([30, 39], (1, 1, entry))
        assert status == pp.PP_PAGED_BAD_PAGE and not bool((out[0] == 7).any())
    status, out, before, c = run([30, 32], (1, 2, -1))            # the page that the new row wants
    assert status == pp.PP_PAGED_BAD_PAGE
    changed = (c.k_pages != before).flatten(1).any(1)
    assert int(changed.sum()) == 1                     # that of the other prompt's row
    assert run([30, 32], (1, 3, -1))[0] == 0           # a page that nothing wants


@pytest.mark.gpu
def test_steps_after_prefill_match_the_contiguous_step():
    """A run as it is used: prefill, its caches into pages, a few tokens; beside the same over contiguous caches."""
    lengths = np.array([45, 3, 130, 64, 1], np.int32)
    hq, hkv, d, steps = 8, 2, 128, 5
    pre = PrefillBatch(lengths, hq, hkv, d, 10000.0, room=steps + 1)
    pre.load(*(normal((int(lengths.sum()), h, d), s) for s, h in enumerate((hq, hkv, hkv))))
    pre.run_fused()
    caches = PagedCaches.allocate(len(lengths), 30, 200, hkv, d, 16)
    for i, n in enumerate(lengths):
        caches.reserve(i, int(n) + steps)
    ln = caches.append_prefill(pre)
    paged, flat = PagedDecoder(caches, hq, 10000.0), DecodeBatch.from_prefill(pre)
    for s in range(steps):
        q, k, v = new_rows(len(lengths), hq, hkv, d, 50 + s, True)
        a = paged.step(ln, q, k, v)
        b = flat.step(*(x.contiguous() for x in (q, k, v)))
        ln += 1
        e = (a.float() - b.float()).abs()
        assert float(e.max()) <= MAX_ABS_TOL and float(e.mean()) <= MEAN_ABS_TOL
    assert paged.device_status() == 0 and int(caches.status) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("shared", [False, True])
def test_captured_step_follows_the_lengths(shared):
    """One captured step (append, attention, the lengths' increment), replayed while prompts grow over chunk and page borders and
    one leaves; another graph of its own decoder runs on a second stream meanwhile."""
    hq, hkv, d, page = 4, 2, 64, 16
    start = np.array([32, 47, 63, 40], np.int32)
    common = [0, (0, 2), (0, 2), 0] if shared else None

    def make(seed):
        P = Pages(start + 45, hkv, d, page, False, BF16, seed=seed, common=common)
        c = P.cuda()
        ln = torch.from_numpy(start).cuda()
        groups = (torch.tensor([0, 3], dtype=torch.int32, device="cuda"), torch.tensor([32], dtype=torch.int32, device="cuda")) if shared else None
        q, k, v = (x.clone() for x in new_rows(4, hq, hkv, d, seed, False))
        dec = PagedDecoder(c, hq, 10000.0)
        out = torch.zeros(4, hq, d, dtype=BF16, device="cuda")
        return P, c, ln, groups, q, k, v, dec, out

    def body(m):
        _, c, ln, groups, q, k, v, dec, out = m
        dec.step(ln, q, k, v, out=out, groups=groups)
        ln.add_((ln >= 0).to(torch.int32))

    graphs, eager = [], [make(21), make(22)]
    for seed in (21, 22):
        m = make(seed)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            body(m)                                    # warm-up (allocates the workspace)
        s.synchronize()
        m[2].copy_(torch.from_numpy(start))
        for pool, x in zip((m[1].k_pages, m[1].v_pages), m[0].pools):
            pool.copy_(x)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            body(m)
        graphs.append((g, m, s))
    torch.cuda.synchronize()
    for step in range(40):
        for (g, m, s), e in zip(graphs, eager):
            new = new_rows(4, hq, hkv, d, 1000 + step, False)
            for dst in (m, e):
                for x, y in zip(dst[4:7], new):
                    x.copy_(y)
                if step == 30:
                    dst[2][3] = -1
        torch.cuda.synchronize()
        for g, m, s in graphs:
            with torch.cuda.stream(s):
                g.replay()
        for e in eager:
            body(e)
        torch.cuda.synchronize()
        for (g, m, s), e in zip(graphs, eager):
            assert torch.equal(m[8], e[8]) and torch.equal(m[2], e[2]), step
            assert torch.equal(m[1].k_pages, e[1].k_pages) and torch.equal(m[1].v_pages, e[1].v_pages)
            assert m[7].device_status() == 0


@pytest.mark.gpu
def test_step_on_another_stream_and_twice_the_same():
    lengths = np.array([100, 900, 0, 17] * 30, np.int32)
    P = Pages(lengths, 4, 128, 32, True, BF16, seed=14)
    c = P.cuda()
    q = new_rows(len(lengths), 8, 4, 128, 15, True)[0]
    ln = torch.from_numpy(lengths).cuda()
    first = PagedDecoder(c, 8, 10000.0).step(ln, q)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        dec = PagedDecoder(c, 8, 10000.0)
        for _ in range(5):
            second = dec.step(ln, q)
    s.synchronize()
    assert torch.equal(first, second)


# ------------------------------------------------------------------------------------------
# GPU: shared rows
# ------------------------------------------------------------------------------------------
def shared_case(groups, hq, hkv, d, page, rows_first, fresh, seed, poison=True, outside=()):
    """groups: (rows shared, rows in all of every prompt). Prompts of `outside` come last. Lengths < 0: rows of no prompt."""
    lengths, common, ptr, shared = [], [], [0], []
    for rows, members in groups:
        lead = None
        for n in members:
            i = len(lengths)
            lengths.append(n)
            if n < 0:
                common.append(0)
            elif lead is None:
                lead = i
                common.append(0)
            else:
                common.append((lead, max(min(rows, n, lengths[lead]), 0) // page))
        ptr.append(len(lengths))
        shared.append(rows)
    lengths += list(outside)
    common += [0] * len(outside)
    lengths = np.array(lengths, np.int32)
    # (of a group with a short prompt the pages are shared as far as that one goes)
    for g, (rows, members) in enumerate(groups):
        least = min([rows] + [n for n in members if n >= 0])
        for i in range(ptr[g], ptr[g + 1]):
            if isinstance(common[i], tuple):
                common[i] = (common[i][0], max(least, 0) // page)
    P = Pages(np.maximum(lengths, -1) + fresh, hkv, d, page, rows_first, BF16, seed=seed, common=common)
    if poison:
        P.poison(lengths)
    to = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    return P, lengths, (to(ptr), to(shared))


# P and the queries are rounded to bf16 for the shared rows. A rounding of a query moves a score by up to 2^-8 sum|q k| scale, about
# 2^-8 / sqrt(3) in the mean square for N(0, 1) elements at 1 / sqrt(d), that of a weight the weight by up to 2^-8: together below
# half a hundredth of |v - O|, in all directions, and O itself is rounded: the tolerances of the prefill, whose roundings these are.
LOOSE = (MAX_ABS_TOL, MEAN_ABS_TOL)


@pytest.mark.gpu
@pytest.mark.parametrize("fresh", [True, False])
@pytest.mark.parametrize("groups,hq,hkv,d,page,rows_first,outside", [
    ([(64, [70, 64, 100])], 4, 4, 128, 16, False, ()),
    ([(512, [512 + 3 * i for i in range(20)])], 8, 2, 128, 64, True, ()),
    ([(333, [340, 350, 333])], 8, 1, 64, 32, False, (5, 0, -1, 77)),                     # not whole pages; prompts of no group
    ([(128, [130, 200]), (0, [5, 9]), (640, [700, 650, 1000]), (16, [16, 20, 40, 17])], 4, 2, 128, 16, True, ()),
    ([(256, [300, -1, 280, -1]), (256, [-1, -1]), (64, []), (256, [256])], 6, 2, 64, 256, False, ()),   # idle rows, an idle and an empty group
    ([(1000, [200, 900, 1000])], 4, 4, 64, 16, False, ()),                               # longer than the shortest prompt
    ([(2000, [2000 + i for i in range(70)])], 8, 1, 128, 128, True, ()),                 # 560 query rows: three tile pairs
    ([(4096, [4100] * 2)], 2, 1, 64, 32, True, ()),
    ([(32 * i, [32 * i + 1 + j for j in range(3)]) for i in range(1, 40)], 2, 2, 64, 16, False, ()),    # more items than CTAs have pieces
])
def test_shared_step(groups, hq, hkv, d, page, rows_first, outside, fresh):
    P, lengths, g = shared_case(groups, hq, hkv, d, page, rows_first, fresh, seed=len(groups) + d, outside=outside)
    caches = P.cuda()
    q, k, v = new_rows(len(lengths), hq, hkv, d, 31, True)
    args = (k, v) if fresh else (None, None)
    before = [x.clone() for x in P.pools]
    out = torch.full((len(lengths), hq, d), 7.0, dtype=BF16, device="cuda")
    dec = PagedDecoder(caches, hq, 10000.0)
    dec.step(torch.from_numpy(lengths).cuda(), q, *args, out=out, groups=g)
    assert dec.device_status() == 0
    assert bool((out[torch.from_numpy(lengths < 0).cuda()] == 7).all())
    check_step(P, lengths, q, *args, out, before, 10000.0, loose=LOOSE)


@pytest.mark.gpu
def test_shared_step_of_a_long_prefix():
    """16384 shared rows for 40 prompts: one group of several tile pairs cut into pieces, scores whose maximum moves late."""
    groups = [(16384, [16384 + 5 * i for i in range(40)])]
    P, lengths, g = shared_case(groups, 8, 2, 128, 64, False, True, seed=77, poison=False)
    at = torch.from_numpy(P.table[0, 16000 // 64:16384 // 64].astype(np.int64))
    P.pools[0][at] = (P.pools[0][at].float() * 4).to(BF16)         # scores of up to 4 * 4.5 log2 units above the ones before
    caches = P.cuda()
    q, k, v = new_rows(len(lengths), 8, 2, 128, 33, False)
    before = [x.clone() for x in P.pools]
    dec = PagedDecoder(caches, 8, 500000.0)
    ln = torch.from_numpy(lengths).cuda()
    out = dec.step(ln, q, k, v, groups=g)
    assert dec.device_status() == 0
    alone = dec.step(ln, q, k, v)
    # Keys four times as large: a query's rounding moves a score four times as far, and fewer keys carry the sum.
    e = (out.float() - alone.float()).abs()
    assert float(e.max()) <= 4 * MAX_ABS_TOL and float(e.mean()) <= 4 * MEAN_ABS_TOL
    check_step(P, lengths[:3], q[:3], k[:3], v[:3], alone[:3], [_with_rows(b, a, P, lengths, 3) for b, a in zip(before, (caches.k_pages, caches.v_pages))], 500000.0)


def _with_rows(before, after, P, lengths, first):
    """`before` with the new rows of the prompts from `first` on."""
    after = after.cpu()
    for i in range(first, len(lengths)):
        page, row = int(P.table[i, lengths[i] // P.page]), int(lengths[i]) % P.page
        before[page, :, row] = after[page, :, row]
    return before


@pytest.mark.gpu
def test_shared_step_says_what_is_wrong():
    P, lengths, (ptr, shared) = shared_case([(64, [70, 64, 100]), (32, [40, 50])], 4, 4, 64, 16, False, False, seed=6)
    caches = P.cuda()
    q = new_rows(5, 4, 4, 64, 7, False)[0]
    ln = torch.from_numpy(lengths).cuda()
    ref = PagedDecoder(caches, 4, 10000.0).step(ln, q)
    for bad in ([0, 6, 5], [3, 1, 5], [-1, 3, 5], [0, 2, 2 ** 31 - 1]):
        dec = PagedDecoder(caches, 4, 10000.0)
        out = dec.step(ln, q, groups=(torch.tensor(bad, dtype=torch.int32, device="cuda"), shared))
        assert dec.device_status() == pp.PP_PAGED_BAD_GROUPS
        assert torch.equal(out, ref)                   # nothing was shared
    dec = PagedDecoder(caches, 4, 10000.0)
    caches.page_table[0, 1] = 99                       # the row that stands for the group's
    out = dec.step(ln, q, groups=(ptr, shared))
    assert dec.device_status() == pp.PP_PAGED_BAD_PAGE and torch.equal(out[3:], dec.step(ln, q, groups=(ptr, shared))[3:])
    dec = PagedDecoder(caches, 4, 10000.0)
    out = dec.step(ln, q, groups=(ptr, torch.tensor([-5, -2 ** 31], dtype=torch.int32, device="cuda")))
    assert torch.equal(out[3:], ref[3:])               # negative: nothing is shared


@pytest.mark.gpu
def test_samples_of_one_prompt():
    """Parallel sampling as it is used: one prefill, its whole pages shared by all samples and the rest appended to each, a few steps."""
    hq, hkv, d, page, samples, steps = 8, 2, 64, 16, 6, 4
    n = 107
    pre = PrefillBatch([n], hq, hkv, d, 10000.0)
    pre.load(*(normal((n, h, d), s) for s, h in enumerate((hq, hkv, hkv))))
    pre.run_fused()
    caches = PagedCaches.allocate(samples, 40, 160, hkv, d, page)
    caches.reserve(0, n + steps)
    caches.append_prefill(pre)
    tail = n - n // page * page
    for i in range(1, samples):
        assert caches.share(0, i, n) == n - tail
        caches.reserve(i, n + steps)
        at = torch.arange(n - tail, n, dtype=torch.int32, device="cuda")
        caches.append(torch.full_like(at, i), at, pre.kk.view(-1, hkv, d)[:n][-tail:], pre.v.view(-1, hkv, d)[:n][-tail:], 10000.0, rotated=True)
    ln = torch.full((samples,), n, dtype=torch.int32, device="cuda")
    g = (torch.tensor([0, samples], dtype=torch.int32, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda"))
    dec = PagedDecoder(caches, hq, 10000.0)
    for s in range(steps):
        q, k, v = new_rows(samples, hq, hkv, d, 90 + s, False)
        out = dec.step(ln, q, k, v, groups=g)
        ln += 1
        alone = dec.step(ln, q)                        # (the same query at the same position: the row is there now)
        e = (out.float() - alone.float()).abs()
        assert float(e.max()) <= MAX_ABS_TOL and float(e.mean()) <= MEAN_ABS_TOL
    assert dec.device_status() == 0 and int(caches.status) == 0


# ------------------------------------------------------------------------------------------
# Calls at the edges
# ------------------------------------------------------------------------------------------
def test_pages_of_prompts_that_there_are_not():
    c = PagedCaches.allocate(3, 8, 64, 1, 64, page_size=16, device="cpu")
    c.reserve(0, 40)
    for call in (lambda: c.reserve(-1, 16), lambda: c.reserve(3, 16), lambda: c.share(-3, 1, 16), lambda: c.share(0, 3, 16), lambda: c.release(-1)):
        with pytest.raises(IndexError):
            call()
    before = c.page_table.clone()
    assert c.share(0, 1, -20) == 0 and torch.equal(c.page_table, before)
    c.reserve(1, 16)                                   # the prompt was left empty, and the free pages as they were
    assert int(c.page_table[1][0]) not in c.page_table[0][:3].tolist()


def test_pools_are_allocated_as_zeros():
    for dtype in (BF16, E4M3):
        scales = {} if dtype is BF16 else {"k_scale": torch.ones(2), "v_scale": torch.ones(2)}
        c = PagedCaches.allocate(1, 3, 40, 2, 64, page_size=16, dtype=dtype, device="cpu", **scales)
        assert c.k_pages.dtype is dtype and c.k_pages.shape == (3, 2, 16, 64) and not bool(c.k_pages.float().any() or c.v_pages.float().any())


@pytest.mark.gpu
def test_workspaces_of_a_growing_batch_stay_bounded():
    hq, hkv, d = 2, 1, 64
    caches = PagedCaches.allocate(200, 200, 16, hkv, d, 16)
    for i in range(200):
        caches.reserve(i, 16)
    dec = PagedDecoder(caches, hq, 10000.0)
    for k in range(1, 201):
        q, kn, vn = new_rows(k, hq, hkv, d, k, False)
        dec.step(torch.zeros(k, dtype=torch.int32, device="cuda"), q, kn, vn)
    assert dec.device_status() == 0
    sizes = [b for _, b in dec._workspaces]
    assert sum(sizes) <= 2 * sizes[-1] and sizes[-1] <= 2 * pp.pp_paged_decode_workspace_bytes(dec.params, 200, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("shared", [False, True])
def test_nothing_is_read_from_a_workspace_that_was_not_written(shared):
    """The same step over a workspace of zeros and over one whose numbers are all NaN, with rows of no prompt inside a group."""
    hq, hkv, d, page = 8, 2, 128, 16
    lengths = np.array([70, -1, 90, 64, 0, 130, -1, 300], np.int32)
    caches = PagedCaches.allocate(len(lengths), 90, 330, hkv, d, page)
    caches.reserve(0, 71)
    for i in range(1, len(lengths)):
        if i in (2, 3):
            caches.share(0, i, 64)
        if lengths[i] >= 0:
            caches.reserve(i, int(lengths[i]) + 1)
    caches.k_pages.normal_()
    caches.v_pages.normal_()
    ln = torch.from_numpy(lengths).cuda()
    q, k, v = new_rows(len(lengths), hq, hkv, d, 5, False)
    groups = (torch.tensor([0, 4, 6], dtype=torch.int32, device="cuda"), torch.tensor([64, 0], dtype=torch.int32, device="cuda")) if shared else None
    dec = PagedDecoder(caches, hq, 10000.0)
    outs = []
    dec.step(ln, q, k, v, groups=groups)
    for byte in (0, 255):
        dec._workspaces[-1][0].fill_(byte)
        out = torch.full((len(lengths), hq, d), 7.0, dtype=BF16, device="cuda")
        outs.append(dec.step(ln, q, k, v, out=out, groups=groups).cpu())
    assert dec.device_status() == 0 and torch.equal(*outs)
    assert bool((outs[0][1] == 7).all() and (outs[0][6] == 7).all()) and bool(torch.isfinite(outs[0]).all())


@pytest.mark.gpu
def test_no_groups_is_the_step_without_them():
    hq, hkv, d = 4, 2, 64
    caches = PagedCaches.allocate(2, 8, 40, hkv, d, 16)
    for i in range(2):
        caches.reserve(i, 30)
    caches.k_pages.normal_()
    caches.v_pages.normal_()
    ln = torch.tensor([20, 29], dtype=torch.int32, device="cuda")
    q, _, _ = new_rows(2, hq, hkv, d, 9, False)
    dec = PagedDecoder(caches, hq, 10000.0)
    none = (torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert torch.equal(dec.step(ln, q), dec.step(ln, q, groups=none))


@pytest.mark.gpu
@pytest.mark.parametrize("shared", [False, True])
def test_step_of_the_most_prompts(shared):
    """8192 prompts, and with shared rows 4096 groups of two: every row against the float64 form."""
    hq, hkv, d, page, k = 2, 1, 64, 16, 8192
    g = torch.Generator(device="cuda").manual_seed(3)
    n_pages = k // 2 + k
    caches = PagedCaches.allocate(1, n_pages, 16, hkv, d, page)
    table = torch.empty((k, 2), dtype=torch.int32, device="cuda")
    table[:, 0] = torch.arange(k, device="cuda", dtype=torch.int32) // 2
    table[:, 1] = k // 2 + torch.arange(k, device="cuda", dtype=torch.int32)
    pools = [torch.randn((n_pages, hkv, page, d), device="cuda", dtype=BF16, generator=g) for _ in range(2)]
    caches = PagedCaches(*pools, table)
    lengths = torch.randint(16, 33, (k,), dtype=torch.int32, device="cuda", generator=g)
    q = torch.randn((k, hq, d), device="cuda", dtype=BF16, generator=g)
    groups = (2 * torch.arange(k // 2 + 1, dtype=torch.int32, device="cuda"), torch.full((k // 2,), 16, dtype=torch.int32, device="cuda")) if shared else None
    dec = PagedDecoder(caches, hq, 10000.0)
    out = dec.step(lengths, q, groups=groups)
    assert dec.device_status() == 0
    rows = [x[table.long()][:, :, 0].reshape(k, 2 * page, d).double() for x in pools]
    turned = torch.from_numpy(rotate64(host64(q), lengths.cpu().numpy() - 1, 10000.0)).cuda()
    s = torch.einsum("khd,krd->khr", turned, rows[0]) / math.sqrt(d)
    s = s.masked_fill(torch.arange(2 * page, device="cuda")[None, None, :] >= lengths[:, None, None], -math.inf)
    p = torch.softmax(s, -1)
    want = torch.einsum("khr,krd->khd", p, rows[1])
    # O is rounded to bf16 once: 2^-8 of it. A query reaches the products as two bf16 numbers (2^-16 of it), over shared rows as one
    # (2^-8); 2^-17 for the rotation and a sum of 64 products in fp32. That moves a score by at most e = (that) sum |q k| scale, and so
    # a weight over the sum of them by a factor of exp(2 e) at most. A weight is one bf16 number over shared rows (2^-8 of it),
    # else two, the first of them cut (2^-7 2^-8); 2^-17 for the sums over at most 33 rows in fp32. All of it times sum p |v|.
    q_part, p_part = (2.0 ** -8, 2.0 ** -8) if shared else (2.0 ** -16, 2.0 ** -15)
    e = torch.einsum("khd,krd->khr", turned.abs(), rows[0].abs()).amax(-1, keepdim=True) / math.sqrt(d) * (q_part + 2.0 ** -17)
    err = torch.einsum("khr,krd->khd", p, rows[1].abs()) * (torch.exp(2 * e) - 1 + p_part + 2.0 ** -17) * (1 + p_part)
    tol = want.abs() * 2.0 ** -8 + err * (1 + 2.0 ** -8)
    assert bool(((out.double() - want).abs() <= tol).all())


def _random_caches(lengths, room, hkv, d, page, shared_pages=0):
    """Caches of random contents whose prompts begin with the same pages."""
    n = len(lengths)
    caches = PagedCaches.allocate(n, n * -(-room // page), room, hkv, d, page)
    caches.reserve(0, room)
    for i in range(1, n):
        caches.share(0, i, shared_pages * page)
        caches.reserve(i, room)
    caches.k_pages.normal_()
    caches.v_pages.normal_()
    return caches


@pytest.mark.gpu
@pytest.mark.parametrize("shared", [False, True])
def test_steps_queued_one_behind_the_other_are_the_steps_alone(shared):
    """Kernels of neighbouring calls overlap; what each of them reads must be there all the same. Appends, steps and changes of the
    lengths, queued without a pause, against the same calls with a synchronisation after each."""
    hq, hkv, d, page, n, steps = 8, 2, 128, 16, 12, 40
    lengths = np.arange(n, dtype=np.int32) * 37 + 70
    groups = (torch.tensor([0, 8, n], dtype=torch.int32, device="cuda"), torch.tensor([64, 48], dtype=torch.int32, device="cuda")) if shared else None
    torch.manual_seed(11)
    first = _random_caches(lengths, 600, hkv, d, page, 4)
    state = first.k_pages.clone(), first.v_pages.clone()
    new = [new_rows(n, hq, hkv, d, 100 + s, False) for s in range(steps)]
    extra = [new_rows(n, hq, hkv, d, 200 + s, False) for s in range(steps)]
    every = torch.arange(n, dtype=torch.int32, device="cuda")

    def run(pause):
        first.k_pages.copy_(state[0])
        first.v_pages.copy_(state[1])
        dec, ln, outs = PagedDecoder(first, hq, 10000.0), torch.from_numpy(lengths).cuda(), []
        torch.cuda.synchronize()
        for s in range(steps):
            q, k, v = new[s]
            outs.append(dec.step(ln, q, k, v, groups=groups))
            if pause:
                torch.cuda.synchronize()
            ln += 1
            if s % 3 == 0:                             # a row more, by the other call
                first.append(every, ln, extra[s][1], extra[s][2], 10000.0)
                ln += 1
            if pause:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert dec.device_status() == 0 and int(first.status) == 0
        return torch.stack(outs), first.k_pages.clone(), first.v_pages.clone()

    for a, b in zip(run(True), run(False)):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_steps_on_two_streams_at_once():
    hq, hkv, d, page, n = 8, 2, 64, 32, 20
    lengths = np.arange(n, dtype=np.int32) * 53 + 130
    torch.manual_seed(12)
    caches = _random_caches(lengths, 1200, hkv, d, page, 4)
    ln = torch.from_numpy(lengths).cuda()
    groups = (torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.tensor([128], dtype=torch.int32, device="cuda"))
    qs = [new_rows(n, hq, hkv, d, 300 + s, False)[0] for s in range(2)]
    want = [PagedDecoder(caches, hq, 10000.0).step(ln, qs[0]), PagedDecoder(caches, hq, 10000.0).step(ln, qs[1], groups=groups)]
    torch.cuda.synchronize()
    streams, decs = [torch.cuda.Stream() for _ in range(2)], [PagedDecoder(caches, hq, 10000.0) for _ in range(2)]
    outs = [[], []]
    for _ in range(30):
        for x in range(2):
            with torch.cuda.stream(streams[x]):
                outs[x].append(decs[x].step(ln, qs[x], groups=groups if x else None))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[x]) for x in range(2) for o in outs[x]) and decs[0].device_status() == decs[1].device_status() == 0
