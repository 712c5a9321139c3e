"""The paged cache where it can go wrong, against plain float64 forms."""
import numpy as np
import pytest
import torch

from paper_2404_09529_b200.runner import PagedDecoder
from test_paged import BF16, E4M3, Pages, check_step, new_rows


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
