"""hero_kv_attn where the scores make it hard (K scales of either sign, probabilities far below the largest, scores that fp32 holds in
steps of more than 1), against 64 bits on the same codes and scales."""
import numpy as np
import pytest
import torch

import kv_reference as R
from paper_2310_17723_amd import binding as HB
from test_gpu_kv_attn import TILES, _attend, _check, _filled
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


@pytest.mark.parametrize("S", [1, 40, 140])
@pytest.mark.parametrize("nats", [18.5, 19.75, 20.0])                     # 2^-26.7, 2^-28.5, 2^-28.9 of the largest
@pytest.mark.parametrize("hp", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_a_flat_tail_far_below_the_largest(hero, fmt, hp, nats, S):
    """One key holds nearly all of a row's weight and its V is zero: the result is a long tail of equal probabilities down to 2^-29 of the largest, which are
    normal numbers of FP16 there, off by 2^-11.  The large key is seen first (each later step is taken against its maximum), in the middle, last, and in steps
    that double it."""
    H, Dh, block, L = 1, 64, 16, 480
    p = _filled(hero, fmt, 4, H, Dh, block, L // block)
    q, k = (torch.zeros((4, n, H, Dh), device="cuda") for n in (S, L))
    v = _rows(111, 4, L, H, Dh, torch.float32, spread=False).abs() * 2.0 ** 10
    q[..., 0] = 8
    for b, at in ((0, 3), (1, 250), (2, L - 1), (3, L - 1)):
        k[b, at, :, 0] = nats                                             # the score: 8 nats / sqrt(64)
        v[b, at] = 0
    k[3, 7::40, :, 0] = torch.arange(1, 13, device="cuda")[:, None].float() * 1.25
    v[3, 7::40] = 0
    p.write(k.to(HP[hp]), v.to(HP[hp]), [L] * 4)
    for tile in TILES:
        _check(p, q.to(HP[hp]), Dh ** -0.5, HB.MASK_NONE, [L] * 4, tile=tile)


@pytest.mark.parametrize("S", [1, 40, 140])
@pytest.mark.parametrize("power", [16, 20, 22, 23, 24, 25, 26, 27, 28, 31, 40, 90])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_scores_far_from_zero(hero, fmt, power, S):
    """Scores of 2^16 .. 2^90, where fp32 holds them in steps of up to 2^67: the key of the largest one has all the weight, and the result is its V; it is the
    first, in the middle or the last, the others lie far below it or (one sequence) all scores are below zero.  P is a power of two or off by 2^-11, the denominator is not
    rounded (2^-20 for its reciprocal and the exponentials), the result by half a step of BF16."""
    H, Dh, block, L = 1, 64, 16, 320
    p = _filled(hero, fmt, 5, H, Dh, block, L // block)
    k, v = torch.zeros((5, L, H, Dh), device="cuda"), _rows(121, 5, L, H, Dh, torch.bfloat16, spread=False)
    q = torch.zeros((5, S, H, Dh), device="cuda")
    q[..., 0] = 2.0 ** (power // 2) * (1 + torch.arange(S, device="cuda") % 5 / 8)[:, None]
    at = [0, 3, 170, L - 1, 100]
    for b, i in enumerate(at):
        k[b, i, :, 0] = 1.75 * 2.0 ** (power - power // 2)
    k[4, :, :, 0] -= 2.0 ** (power - power // 2 + 1)                      # -0.25 (100) or -2 times 2^power
    p.write(k.to(torch.bfloat16), v, [L] * 5)
    for tile in TILES:
        y = _attend(p, q.to(torch.bfloat16), 1.0, HB.MASK_NONE, [L] * 5, tile=tile).double().cpu().numpy().reshape(5, S, Dh)
        for b, i in enumerate(at):
            ref = R.rows_of(p.codes["v"], p.scale["v"], p.table, b, L, fmt)[0][i, 0]
            assert (np.abs(y[b] - ref) <= (2.0 ** -11 + 2.0 ** -20 + 2.0 ** -8) * np.abs(ref)).all(), (tile, b, y[b, :, :4], ref[:4])
