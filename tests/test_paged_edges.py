"""The paged cache where it can go wrong, against plain float64 forms."""
import numpy as np
import pytest
import torch

from paper_2404_09529_b200.runner import PagedDecoder
from test_paged import BF16, E4M3, Pages, check_step, host64, new_rows


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
