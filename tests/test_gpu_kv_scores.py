"""hero_kv_attn where the scores make it hard: K scales of either sign, against 64 bits on the same codes and scales."""
import numpy as np
import pytest
import torch

from paper_2310_17723_amd import binding as HB
from test_gpu_kv_attn import TILES, _check, _filled
from test_gpu_kv_cache import HP, _rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S", [1, 40, 140, 300])
@pytest.mark.parametrize("block", [16, 64])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_k_scales_of_either_sign(hero, fmt, block, S):
    """A cache from elsewhere may hold K = codes * scale with a negative scale.  Scores of about -60 .. 60 (in powers of two), so that exponentials against a maximum
    that is not the row's would not fit FP16."""
    H, Dh, L = 2, 64, 512
    p = _filled(hero, fmt, 2, H, Dh, block, L // block, paged=True)
    k, v = (_rows(s, 2, L, H, Dh, torch.bfloat16, spread=False) for s in (101, 102))
    p.write(k, v, [L] * 2)
    sign = np.random.default_rng(103).choice([-1, 1], p.scale["k"].shape).astype(np.float32)
    sign[p.table[1]] = -1                                                 # one sequence: every scale negative
    p.scale["k"] *= sign
    p.dev_scale["k"].copy_(torch.from_numpy(p.scale["k"]))
    q = (_rows(104, 2, S, H, Dh, torch.float32, spread=False) * 12).to(torch.bfloat16)
    for tile in TILES:
        for mask in (HB.MASK_NONE, HB.MASK_CAUSAL):
            _check(p, q, Dh ** -0.5, mask, [L, L - 7], tile=tile)
