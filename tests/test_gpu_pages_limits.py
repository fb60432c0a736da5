"""Paged 8-bit caches at the limits of what their sizes may be."""
import numpy as np
import pytest
import torch

import test_gpu_pages as T
from paper_2601_20357_b200 import binding as TB

pytestmark = pytest.mark.gpu


def test_append_at_the_end_of_the_longest_table_with_the_largest_max_new():
    """Positions up to 2^31 - 257, and as many tokens announced: block numbers times page_tokens pass 2^31 behind the last block."""
    ps, Hkv, hd, blocks = 128, 1, 32, (1 << 24) - 2
    table = torch.full((1, blocks), -1, dtype=torch.int32, device=T.DEV)
    table[0, 0], table[0, -1] = 2, 0
    shape = (1, 3, Hkv, ps, hd)
    p = TB.Pages(k=torch.zeros(shape, dtype=torch.uint8, device=T.DEV), v=torch.zeros(shape, dtype=torch.uint8, device=T.DEV), k_scale=torch.ones(shape[:3], device=T.DEV),
                 v_scale=torch.ones(shape[:3], device=T.DEV), table=table, ref=T.ints([1, 0, 1]))
    x = torch.from_numpy(np.random.default_rng(0).standard_normal((2, 5, Hkv, hd))).to(T.DEV, torch.bfloat16)
    p.append(0, x[0], x[1], None, T.ints([0, 5]), T.ints([ps - 5]), 5)
    p.append(0, x[0], x[1], None, T.ints([0, 5]), T.ints([blocks * ps - 5]), blocks * ps)
    assert p.last_error() == 0
    assert torch.equal(p.k[0, 0], p.k[0, 2]) and torch.equal(p.v[0, 0], p.v[0, 2]) and not p.k[0, 1].any()
    assert p.k[0, 0, 0, -5:].any() and torch.equal(p.k_scale[0, 0], p.k_scale[0, 2]) and torch.equal(p.v_scale[0, 0], p.v_scale[0, 2])
    p.append(0, x[0], x[1], None, T.ints([0, 5]), T.ints([blocks * ps - 4]), blocks * ps)
    assert p.last_error() == TB.ERR_KV_OVERFLOW
