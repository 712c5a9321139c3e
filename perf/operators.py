"""The operators over a paged KV cache by which their speed is judged: rows appended to pages with the position
rotation applied on the way, the generation step over pages, and that step for prompts that share their first pages.

A case is a dict of plain values:
    kind     "append" | "decode" | "shared"
    type     "bf16" | "e4m3": what the pages hold (e4m3: value / scale of the KV head)
    page     rows of a page
    layout   "heads": pools [page, KV head, row, D]; "rows": pools [page, row, KV head, D]
    hq, hkv, d, base, scale
             attention-layer shape, rotary base, softmax scale (0 = 1 / sqrt(d))
    strided  True: q, k, v are slices of one tensor [rows, (hq + 2 hkv) d], as a fused projection leaves them
    prompts, dist, lo, hi, p0, p1, lengths_seed
             append: new rows of each prompt; decode: tokens that each prompt has in its pages (see `_lengths`)
    start    append: every prompt has 0 .. start rows in its pages already
    rotated  append: the keys carry the rotation already (as the prefill leaves them): they are copied
    pad      append: rows of no prompt between the prompts' rows, as in bins whose tails are padded
    fresh    decode, shared: the step brings the new token's key and value, which are appended; otherwise they are
             in the pages already
    idle     decode: rows of a padded batch that belong to no prompt (their length is -1, their output stays)
    groups, samples, shared_lo, shared_hi
             shared: groups of `samples` prompts whose first rows are the same pages; lo .. hi rows of their own
"""
import math

import numpy as np
import torch

own = False

_MHA7B = {"hq": 32, "hkv": 32, "d": 128, "base": 10000.0, "scale": 0.0}
_GQA8B = {"hq": 32, "hkv": 8, "d": 128, "base": 500000.0, "scale": 0.0}
_SHORT = {"hq": 32, "hkv": 8, "d": 64, "base": 500000.0, "scale": 0.0}
_MEDIAN200 = {"dist": "lognormal", "lo": 8, "hi": 2048, "p0": 200.0, "p1": 0.8, "lengths_seed": 0}
_TWO = {"dist": "two_uniform", "lo": 20, "hi": 4000, "p0": 200.0, "p1": 1000.0, "lengths_seed": 0}


def listed():
    append = {"kind": "append", "start": 0, "rotated": False, "pad": 0, "strided": False}
    decode = {"kind": "decode", "fresh": True, "idle": 0, "strided": False}
    shared = {"kind": "shared", "fresh": True, "strided": False, "type": "bf16", "lengths_seed": 0}
    return [
        # one new row for each of 64 prompts of a 7B layer, out of the fused projection: latency
        {"name": "append_step_7b", **append, "type": "bf16", "page": 16, "layout": "heads", "prompts": 64, "dist": "uniform",
         "lo": 1, "hi": 1, "p0": 0.0, "p1": 0.0, "lengths_seed": 0, "start": 2000, "strided": True, **_MHA7B},
        # an ordinary batch's prompts into pages after a prefill that left the keys raw
        {"name": "append_prompts_7b", **append, "type": "bf16", "page": 64, "layout": "rows", "prompts": 64, **_MEDIAN200, **_MHA7B},
        # thousands of short prompts out of padded bins into an 8-bit cache
        {"name": "append_short_e4m3", **append, "type": "e4m3", "page": 16, "layout": "heads", "prompts": 2048, "dist": "pareto",
         "lo": 8, "hi": 8192, "p0": 1.5, "p1": 0.0, "lengths_seed": 0, "pad": 3, **_SHORT},
        # a generation step of nine one-token prompts and a long one: latency
        {"name": "decode_toy", **decode, "type": "bf16", "page": 16, "layout": "heads", "prompts": 10, "dist": "toy", "lo": 1,
         "hi": 1000, "p0": 0.0, "p1": 0.0, "lengths_seed": 0, **_MHA7B},
        # an ordinary batch, multi-head cache, in a graph's padded batch
        {"name": "decode_7b", **decode, "type": "bf16", "page": 64, "layout": "rows", "prompts": 64, **_MEDIAN200, "idle": 5,
         "strided": True, **_MHA7B},
        # a large serving batch, grouped-query heads, small pages
        {"name": "decode_8b_gqa", **decode, "type": "bf16", "page": 16, "layout": "heads", "prompts": 256, **_TWO, **_GQA8B},
        # the same in 8 bits
        {"name": "decode_8b_gqa_e4m3", **decode, "type": "e4m3", "page": 32, "layout": "heads", "prompts": 256, **_TWO, **_GQA8B},
        # one prompt whose cache is the whole work: few rows, a long axis
        {"name": "decode_one_long", **decode, "type": "bf16", "page": 128, "layout": "rows", "prompts": 1, "dist": "uniform",
         "lo": 131071, "hi": 131071, "p0": 0.0, "p1": 0.0, "lengths_seed": 0, **_GQA8B, "fresh": False},
        # 16 samples of one prompt, a few tokens each so far
        {"name": "shared_samples16", **shared, "page": 16, "layout": "heads", "groups": 1, "samples": 16, "shared_lo": 2000,
         "shared_hi": 2000, "lo": 1, "hi": 200, **_GQA8B},
        # parallel sampling for a batch of prompts on a multi-head layer
        {"name": "shared_sampling_7b", **shared, "page": 64, "layout": "rows", "groups": 24, "samples": 8, "shared_lo": 200,
         "shared_hi": 2048, "lo": 1, "hi": 250, **_MHA7B, "strided": True},
        # a serving batch behind one system prompt
        {"name": "shared_system_8b", **shared, "page": 32, "layout": "heads", "groups": 1, "samples": 256, "shared_lo": 8200,
         "shared_hi": 8200, "lo": 20, "hi": 500, **_GQA8B},
        # many questions about one long document, narrow heads
        {"name": "shared_document_d64", **shared, "page": 256, "layout": "rows", "groups": 1, "samples": 64, "shared_lo": 32700,
         "shared_hi": 32700, "lo": 8, "hi": 300, **_SHORT, "fresh": False},
    ]


def _spread(rng, case, k):
    lo, hi, dist = case["lo"], case["hi"], case["dist"]
    if dist == "uniform":
        out = rng.integers(lo, hi + 1, size=k)
    elif dist == "lognormal":            # p0 = median, p1 = sigma
        out = np.clip(np.rint(np.exp(np.log(case["p0"]) + case["p1"] * rng.standard_normal(k))), lo, hi)
    elif dist == "pareto":               # p0 = alpha
        out = np.clip(np.floor(lo * (1.0 - rng.random(k)) ** (-1.0 / case["p0"])), lo, hi)
    elif dist == "two_uniform":          # 70 % in [lo, p0], 30 % in [p1, hi]
        u = rng.random(k)
        out = np.where(u < 0.7, rng.integers(lo, int(case["p0"]) + 1, k), rng.integers(int(case["p1"]), hi + 1, k))
    else:                                # "toy": prompts of `lo` tokens and one of `hi`
        out = np.full(k, lo)
        out[-1] = hi
    return out.astype(np.int64)


def _lengths(case):
    """append: (new rows, rows before) of every prompt. decode: tokens in the pages, -1 for idle rows. shared: (tokens in the
    pages of every prompt, shared rows of every group). They belong to the case: every seed has the same work."""
    rng = np.random.default_rng(case["lengths_seed"])
    if case["kind"] == "append":
        new = _spread(rng, case, case["prompts"])
        return new, rng.integers(0, case["start"] + 1, size=len(new))
    if case["kind"] == "decode":
        return np.concatenate([_spread(rng, case, case["prompts"]), np.full(case["idle"], -1, np.int64)])
    shared = rng.integers(case["shared_lo"], case["shared_hi"] + 1, size=case["groups"]) // case["page"] * case["page"]
    mine = rng.integers(case["lo"], case["hi"] + 1, size=(case["groups"], case["samples"]))
    return (shared[:, None] + mine).reshape(-1), shared


def draw(rng):
    """One more case of the same ranges: 1 to 2048 prompts of 0 to 131072 tokens, 1 to 256 samples of up to 32768 shared rows, 4 to
    32 query heads in groups of 1 to 8 (3 among them), both head dimensions, types and layouts, pages of 16 to 256 rows."""
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["append", "decode", "decode", "shared", "shared"])
        hq, hkv = rng.choice([(4, 4), (8, 8), (16, 16), (32, 32), (12, 4), (24, 8), (8, 4), (16, 4), (32, 8), (32, 4), (8, 1)])
        log = lambda a, b: int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))
        case = {"kind": kind, "type": "bf16" if kind == "shared" else rng.choice(["bf16", "bf16", "e4m3"]),
                "page": rng.choice([16, 16, 32, 64, 128, 256]), "layout": rng.choice(["heads", "rows"]), "hq": hq, "hkv": hkv,
                "d": rng.choice([64, 128, 128]), "base": rng.choice([10000.0, 500000.0]), "scale": rng.choice([0.0, 0.0, 0.0, 0.125]),
                "strided": rng.choice([False, True]), "lengths_seed": rng.randrange(1 << 30)}
        if kind == "shared":
            top = log(16, 32768)
            case.update(groups=log(1, 64), samples=log(1, 256), shared_lo=rng.randrange(top + 1), shared_hi=top, lo=rng.randrange(2),
                        hi=log(1, 2000), fresh=rng.choice([True, True, False]))
        else:
            middle = math.exp(rng.uniform(0.0, math.log(65536.0)))
            dist = rng.choice(["uniform", "lognormal", "lognormal", "pareto", "two_uniform"])
            case.update(dist=dist, prompts=log(1, 2048 if kind == "append" else 512), p0=0.0, p1=0.0)
            if dist == "uniform":
                case.update(lo=int(middle / 4), hi=int(middle * 2))
            elif dist == "lognormal":
                case.update(lo=rng.randrange(2), hi=131072, p0=middle, p1=rng.uniform(0.3, 1.2))
            elif dist == "pareto":
                case.update(lo=max(1, int(middle / 2)), hi=131072, p0=rng.uniform(1.2, 2.5))
            else:
                case.update(lo=int(middle / 10), hi=max(2, int(middle * 2)), p0=float(max(2, int(middle))), p1=float(max(2, int(middle))))
            if kind == "append":
                case.update(start=rng.choice([0, log(1, 30000)]), rotated=rng.choice([False, False, True]), pad=rng.choice([0, rng.randrange(8)]))
            else:
                case.update(fresh=rng.choice([True, True, False]), idle=rng.choice([0, rng.randrange(9)]))
        lengths = _lengths(case)
        if kind == "append":
            rows, longest = int(lengths[0].sum()), 0
            held = rows + int(lengths[1].sum())
        else:
            lengths = lengths if kind == "decode" else lengths[0]
            rows, longest = len(lengths), int(lengths.max())
            held = int(lengths.clip(0).sum())
        # (something to do, room for three states, and for the plain form, which pads every prompt to the longest)
        if rows < 1 or (kind != "append" and longest < 1) or held + rows > 1 << 20 or 4 * hkv * case["d"] * max(held, rows * longest) > 12 << 30:
            continue
        if _cost(case) <= 0.8 * most:
            return case


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 8e14


def work(case):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    cell = 2 * d * hkv * (1 if case["type"] == "e4m3" else 2)        # K and V of one row in the pages
    if case["kind"] == "append":
        rows = int(_lengths(case)[0].sum())
        return {"bytes": rows * (4 * d * hkv + cell + 8), "flops": 0 if case["rotated"] else 3 * rows * hkv * d}
    fresh = int(case["fresh"])
    if case["kind"] == "decode":
        lengths = _lengths(case)
        lengths = lengths[lengths >= 0]
        rows = int(lengths.sum())
    else:
        lengths, shared = _lengths(case)
        rows = int(lengths.sum()) - int(shared.sum()) * (case["samples"] - 1)
    k = len(lengths)
    return {"bytes": rows * cell + k * (4 * hq * d + fresh * (4 * hkv * d + cell)), "flops": 4 * hq * d * (int(lengths.sum()) + k * fresh)}


def _normal(shape, g):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _new_rows(case, n, g):
    """q, k, v of n rows: tensors of their own, or slices of one."""
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if not case["strided"]:
        return [_normal((n, h, d), g) for h in (hq, hkv, hkv)]
    whole = _normal((n, hq + 2 * hkv, d), g)
    return [whole[:, :hq], whole[:, hq:hq + hkv], whole[:, hq + hkv:]]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    page, kind = case["page"], case["kind"]
    s = {"case": case}
    # which pages every prompt has: those of its group first, then its own, from anywhere in the pool
    if kind == "append":
        new, before = _lengths(case)
        room = new + before
        common = np.zeros(len(new), np.int64)
    elif kind == "decode":
        lengths = _lengths(case)
        room = lengths.clip(0) + int(case["fresh"]) * (lengths >= 0)
        common = np.zeros(len(lengths), np.int64)
    else:
        lengths, shared = _lengths(case)
        room = lengths + int(case["fresh"])
        common = np.repeat(shared // page, case["samples"])
    count = -(-room // page)
    table = np.full((len(room), int(count.max()) + 1), -1, np.int32)
    groups = shared // page if kind == "shared" else np.zeros(0, np.int64)
    n_pages = int((count - common).sum() + groups.sum()) + 3
    ids = rng.permutation(n_pages).astype(np.int32)
    at = 0
    for i, n in enumerate(groups):
        table[i * case["samples"]:(i + 1) * case["samples"], :n] = ids[at:at + n]
        at += n
    for i, (a, b) in enumerate(zip(common, count)):
        table[i, a:b] = ids[at:at + b - a]
        at += b - a
    s["table"] = torch.from_numpy(table).cuda()
    hkv, d = case["hkv"], case["d"]
    shape = (n_pages, hkv, page, d) if case["layout"] == "heads" else (n_pages, page, hkv, d)
    s["k_pages"], s["v_pages"] = _normal(shape, g), _normal(shape, g)
    s["k_scale"] = s["v_scale"] = None
    if case["type"] == "e4m3":
        # largest magnitudes of about 5 at 0.25 to 0.8 of the type's range
        s["k_scale"], s["v_scale"] = (0.014 + 0.031 * torch.rand(hkv, generator=g, device="cuda") for _ in range(2))
        for x in ("k", "v"):
            head = s[x + "_scale"].view(-1, 1, 1) if case["layout"] == "heads" else s[x + "_scale"].view(-1, 1)
            s[x + "_pages"] = (s[x + "_pages"].float() / head).to(torch.float8_e4m3fn)
    if kind == "append":
        gap = case["pad"]
        prompt = np.concatenate([np.concatenate([np.full(n, i), np.full(gap, -1)]) for i, n in enumerate(new)]).astype(np.int32)
        position = np.concatenate([np.concatenate([b + np.arange(n), np.zeros(gap)]) for n, b in zip(new, before)]).astype(np.int32)
        s["prompt"], s["position"] = torch.from_numpy(prompt).cuda(), torch.from_numpy(position).cuda()
        _, s["k_new"], s["v_new"] = _new_rows(case, len(prompt), g)
        return s
    s["lengths"] = torch.from_numpy(lengths.astype(np.int32)).cuda()
    s["longest"] = int(room.max())
    s["q"], s["k_new"], s["v_new"] = _new_rows(case, len(lengths), g)
    s["o"] = torch.zeros((len(lengths), case["hq"], d), dtype=torch.bfloat16, device="cuda")
    if kind == "shared":
        s["group_ptr"] = torch.arange(case["groups"] + 1, dtype=torch.int32, device="cuda") * case["samples"]
        s["shared_len"] = torch.from_numpy(shared.astype(np.int32)).cuda()
    return s


def _rotate(x, position, base):
    """x [n, heads, d] float32, rotated by its row's position; the angles in 64 bits."""
    half = x.shape[-1] // 2
    theta = base ** (-2.0 * torch.arange(half, device=x.device, dtype=torch.float64) / x.shape[-1])
    angle = position.double()[:, None] * theta
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _cells(pages, layout, page, row):
    """An index of the [.., heads, d] cells of rows of pages."""
    return (page, slice(None), row) if layout == "heads" else (page, row)


def _store(pages, at, x, scale):
    if scale is None:
        pages[at] = x.to(torch.bfloat16)
    else:
        x = (x / scale[:, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
        pages.view(torch.uint8)[at] = x.view(torch.uint8)


def _fetch(pages, at, scale):
    if scale is None:
        return pages[at].float()
    return pages.view(torch.uint8)[at].view(torch.float8_e4m3fn).float() * scale[:, None]


def _append_rows(s, prompt, position, k, v, rotated):
    case = s["case"]
    position = position.long()
    at = _cells(None, case["layout"], s["table"][prompt.long(), position // case["page"]].long(), position % case["page"])
    k = k.float() if rotated else _rotate(k.float(), position, case["base"])
    _store(s["k_pages"], at, k, s["k_scale"])
    _store(s["v_pages"], at, v.float(), s["v_scale"])


def _plain(s):
    case = s["case"]
    if case["kind"] == "append":
        rows = (s["prompt"] >= 0).nonzero()[:, 0]
        _append_rows(s, s["prompt"][rows], s["position"][rows], s["k_new"][rows], s["v_new"][rows], case["rotated"])
        return
    lengths = s["lengths"].long()
    active = lengths >= 0
    if case["fresh"]:
        rows = active.nonzero()[:, 0]
        _append_rows(s, rows, lengths[rows], s["k_new"][rows], s["v_new"][rows], False)
    n = lengths + int(case["fresh"])                    # rows that the query sees; it sits at the last of them
    q = _rotate(s["q"].float(), n - 1, case["base"])
    k, hq, d = q.shape
    hkv = case["hkv"]
    at = torch.arange(s["longest"], device=q.device)
    cells = _cells(None, case["layout"], s["table"][:, at // case["page"]].clamp(min=0).long(), (at % case["page"]).expand(k, -1))
    keys = _fetch(s["k_pages"], cells, s["k_scale"])    # [k, longest, hkv, d]
    scores = torch.einsum("khgd,klhd->khgl", q.view(k, hkv, hq // hkv, d), keys) * (case["scale"] or d ** -0.5)
    del keys
    seen = (at < n[:, None])[:, None, None]
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.where(seen, (scores - top).exp(), 0.0)
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    o = torch.einsum("khgl,klhd->khgd", p, _fetch(s["v_pages"], cells, s["v_scale"])).reshape(k, hq, d)
    s["o"].copy_(torch.where(active[:, None, None], o.to(torch.bfloat16), s["o"]))


def _own(s):
    from paper_2404_09529_b200.runner import PagedCaches, PagedDecoder
    case = s["case"]
    if "caches" not in s:
        s["caches"] = PagedCaches(s["k_pages"], s["v_pages"], s["table"], rows_first=case["layout"] == "rows", k_scale=s["k_scale"],
                                  v_scale=s["v_scale"])
        if case["kind"] != "append":
            s["decoder"] = PagedDecoder(s["caches"], case["hq"], case["base"], softmax_scale=case["scale"])
    if case["kind"] == "append":
        s["caches"].append(s["prompt"], s["position"], s["k_new"], s["v_new"], case["base"], rotated=case["rotated"])
        return
    new = (s["k_new"], s["v_new"]) if case["fresh"] else (None, None)
    groups = (s["group_ptr"], s["shared_len"]) if case["kind"] == "shared" else None
    s["decoder"].step(s["lengths"], s["q"], *new, out=s["o"], groups=groups)


def run(state):
    if own:
        _own(state)
    else:
        _plain(state)
    names = ["k_pages", "v_pages"] if state["case"]["kind"] == "append" else ["o", "k_pages", "v_pages"]
    return {x: state[x] for x in names}


def exact(case, seed):
    """One prompt after another, one row of the pages after another, in 64 bits; a rotation is a complex product."""
    s = prepare(case, seed)
    hq, hkv, d, size = case["hq"], case["hkv"], case["d"], case["page"]
    by_row = case["layout"] == "rows"

    def turned(x, position):                            # x [n, heads, d]
        turn = np.outer(position, [float(case["base"]) ** (-2.0 * j / d) for j in range(d // 2)])
        turn = torch.polar(torch.ones(turn.shape, dtype=torch.float64), torch.from_numpy(turn)).cuda()[:, None]
        x = x.double()
        z = torch.complex(x[..., :d // 2].contiguous(), x[..., d // 2:].contiguous()) * turn
        return torch.cat((z.real, z.imag), -1)

    pools, scales = {}, {}
    for x in "kv":
        p = s[x + "_pages"].to(torch.float64)
        pools[x] = p if by_row else p.transpose(1, 2)   # a view [page, row, head, d]
        scales[x] = 1.0 if s[x + "_scale"] is None else s[x + "_scale"].double()[:, None]
    table = s["table"].cpu().numpy()

    def put(i, position, k, v):
        cell = torch.from_numpy(table[i, position // size].astype(np.int64)).cuda(), torch.from_numpy(position % size).cuda()
        pools["k"][cell] = k / scales["k"]
        pools["v"][cell] = v.double() / scales["v"]

    def out():
        return {x + "_pages": pools[x] if by_row else pools[x].transpose(1, 2) for x in "kv"}

    if case["kind"] == "append":
        prompt, position = s["prompt"].cpu().numpy(), s["position"].cpu().numpy().astype(np.int64)
        rows = np.nonzero(prompt >= 0)[0]
        at = torch.from_numpy(rows).cuda()
        k = s["k_new"][at].double() if case["rotated"] else turned(s["k_new"][at], position[rows])
        put(prompt[rows], position[rows], k, s["v_new"][at])
        return out()
    lengths = s["lengths"].cpu().numpy().astype(np.int64)
    o = torch.zeros((len(lengths), hq, d), dtype=torch.float64, device="cuda")
    held = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[case["type"]]
    for i, n in enumerate(lengths):
        if n < 0:
            continue
        if case["fresh"]:
            # (the row is read back as the pages hold it, rounded)
            k = turned(s["k_new"][i:i + 1], np.array([n]))
            put(np.array([i]), np.array([n]), k, s["v_new"][i:i + 1])
            n += 1
        if n == 0:
            continue
        ids = torch.from_numpy(table[i, :-(-n // size)].astype(np.int64)).cuda()
        rows = {}
        for x in "kv":
            r = pools[x][ids].reshape(-1, hkv, d)[:n].clone()
            r[-1] = r[-1].float().clamp(-448.0, 448.0).to(held).double() if case["type"] == "e4m3" else r[-1].to(held).double()
            rows[x] = (r * scales[x]).transpose(0, 1)   # [hkv, n, d]
        q = turned(s["q"][i:i + 1], np.array([n - 1]))[0].view(hkv, hq // hkv, d)
        w = torch.softmax(q @ rows["k"].transpose(1, 2) * (case["scale"] or 1.0 / math.sqrt(d)), -1)
        o[i] = (w @ rows["v"]).reshape(hq, d)
    return {"o": o, **out()}
