"""hero_kv_write into blocks that another program began with a negative scale: the tokens from before keep their values."""
import numpy as np
import pytest
import torch

import kv_reference as R
from test_gpu_kv_cache import HP, Pool, _rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("small", [True, False])                          # the new tokens: far below the block's largest value, or above it
@pytest.mark.parametrize("hp", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("Dh,block", [(64, 16), (128, 64), (128, 128)])
def test_tokens_behind_a_negative_scale(hero, Dh, block, fmt, hp, small):
    B, H, had, S = 2, 3, block - 5, 3
    p = Pool(hero, fmt, B, H, Dh, block, 2, paged=True, seed=7)
    for x in "kv":
        if fmt == "i8":
            p.codes[x][p.codes[x] == 128] = 129                           # (-128 has no counterpart)
            p.raw[x].copy_(torch.from_numpy(p.codes[x]).cuda().transpose(1, 2))
        p.scale[x][:, 1:] *= -1                                           # head 0 keeps its sign
        p.dev_scale[x].copy_(torch.from_numpy(p.scale[x]))
    before = {x: [R.rows_of(p.codes[x], p.scale[x], p.table, b, had, fmt)[0] for b in range(B)] for x in "kv"}
    new = {x: (_rows(i, B, S, H, Dh, torch.float32, spread=False) * (1e-3 if small else 40.0)).to(HP[hp]) for i, x in enumerate("kv")}
    lens = torch.full((B,), had + S, dtype=torch.int32, device="cuda")
    hero.hero_kv_write(p.cache, new["k"], new["v"], lens)
    for x, got in zip("kv", hero.hero_kv_read(p.cache, had + S, lens, dtype=torch.float32)):
        for b in range(B):
            blk = int(p.table[b, 0])
            scale, old = p.dev_scale[x][blk].cpu().numpy(), np.abs(p.scale[x][blk])
            rows = new[x][b].float().cpu().numpy()
            assert np.array_equal(scale, np.maximum(old, (np.abs(rows).max((0, 2)) / np.float32(R.FORMATS[fmt][1])).astype(np.float32)))
            want, y, s = np.concatenate([before[x][b], rows.astype(np.float64)]), got[b].double().cpu().numpy(), scale.astype(np.float64)[:, None]
            # a code is off by half a step (INT8 1/2; E4M3 2^-4 of the value, 2^-10 below its normal numbers), fl(code s_old), the quotient and code s_new by 2^-24 each
            tol = (s / 2 if fmt == "i8" else np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * s)) + 2.0 ** -22 * np.abs(want)
            assert (np.abs(y - want) <= tol).all(), (x, b, np.argwhere(np.abs(y - want) > tol)[:4])
