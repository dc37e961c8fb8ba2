"""hero_moe_route and hero_moe_combine against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import moe_reference as R
from paper_2310_17723_amd import binding as HB

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _logits(T, E, dt, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((T, E), generator=g) * spread).to(TYPES[dt])


def _check(hero, logits, k, renorm=True, got=None, stride=None):
    T, E = logits.shape
    if got is None:
        d = logits.cuda()
        if stride:
            d = torch.full((T, stride), 1e30, dtype=d.dtype, device="cuda")
            d[:, :E] = logits.cuda()
            d = d[:, :E]
        got = hero.hero_moe_route(d, k, renorm=renorm)
    expert, weight, slot, token, offsets = R.route(logits.float().numpy(), k, renorm)
    names = ("expert", "slot", "row_token", "offsets")
    for name, ref in zip(names, (expert, slot, token, offsets)):
        assert np.array_equal(getattr(got, name).cpu().numpy(), ref), name
    # relative: l - m is rounded once (|l - m| 2^-24 of its exponential), the exponentials are off by 2^-23, the sum of up to E terms by E 2^-24,
    # every term of it by as much as one exponential, the quotient by 2^-24; below 2^-126 numbers are subnormal, off by 2^-149 (or flushed)
    l = np.minimum(logits.float().numpy().astype(np.float64), np.finfo(np.float32).max)
    finite = np.where(np.isfinite(l), l, -np.inf)
    top = finite.max(1, keepdims=True)
    span = np.subtract(top, l, out=np.zeros_like(l), where=np.isfinite(l)).max(initial=0.0)
    bound = weight * (2 * min(span, 110.0) + E + 8) * 2.0 ** -24 + 2.0 ** -126
    w = got.weight.cpu().numpy().astype(np.float64)
    assert (np.abs(w - weight) <= bound).all(), np.max(np.abs(w - weight) / bound)
    assert (w[expert < 0] == 0).all()


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (2, 64, 6), (63, 65, 1), (64, 128, 8), (65, 129, 16), (300, 256, 3), (130, 257, 8), (70, 512, 16), (1000, 4, 4), (1000, 7, 2)])
def test_choices_and_rows(hero, T, E, k, dt):
    for renorm in (True, False):
        _check(hero, _logits(T, E, dt, T + E + k), k, renorm)


def test_ties_go_to_the_lowest_index(hero):
    g = torch.Generator().manual_seed(5)
    for E in (3, 64, 100, 300, 512):
        _check(hero, torch.randint(0, 3, (140, E), generator=g).to(torch.bfloat16), min(E, 6))
    _check(hero, torch.zeros((70, 512)), 16)
    _check(hero, torch.tensor([[0.0, -0.0, 0.0, -0.0]]), 3)                # (equal numbers)


@pytest.mark.parametrize("T", [5, 200])
def test_masked_experts_padding_tokens_infinities_and_nan(hero, T):
    l = _logits(T, 70, "f32", 9)
    l[::3, 10:] = -torch.inf                                              # some experts are out
    l[1::4, :] = -torch.inf                                               # padding
    l[2, :] = torch.nan                                                   # no expert at all
    l[3, ::2] = torch.nan
    l[4, 5], l[4, 69] = torch.inf, torch.inf                              # two experts share the weight
    l[0, 1:], l[0, 0] = -torch.inf, -1e38
    for renorm in (True, False):
        _check(hero, l, 12, renorm)
        _check(hero, torch.full((T, 9), -torch.inf), 3, renorm)
    h = l.clone()
    h[h.abs() < 1e30] *= 100
    _check(hero, h, 12, False)                                            # (weights that are subnormal, and 0)
    _check(hero, l.half(), 12)


def test_large_logits(hero):
    l = _logits(100, 33, "f32", 1) * 1e38
    _check(hero, l, 5)


def test_all_tokens_to_the_same_experts(hero):
    for T in (64, 65, 3000):
        l = _logits(T, 40, "f32", 2)
        l[:, 7] += 100
        l[:, 39] += 90
        _check(hero, l, 2)


def test_rows_of_a_wider_matrix_and_views(hero):
    _check(hero, _logits(100, 37, "bf16", 3), 4, stride=41)
    _check(hero, _logits(1, 37, "f32", 3), 4, stride=64)


def test_many_workgroups(hero):
    """More workgroups of tokens than the scan takes at once (256)."""
    T, E, k = 64 * 300 + 17, 5, 2
    l = _logits(T, E, "f32", 4)
    l[5000:6000] = -torch.inf
    got = hero.hero_moe_route(l.cuda(), k)
    v, i = l.sort(dim=1, descending=True, stable=True)
    flat = torch.where(v[:, :k] > -torch.inf, i[:, :k], E).reshape(-1).numpy()
    order = np.argsort(flat, kind="stable")
    n = int((flat < E).sum())
    slot = np.empty(T * k, np.int64)
    slot[order] = np.arange(T * k)
    assert np.array_equal(got.expert.cpu().numpy().reshape(-1), np.where(flat < E, flat, -1))
    assert np.array_equal(got.slot.cpu().numpy().reshape(-1), np.where(flat < E, slot, -1))
    assert np.array_equal(got.row_token.cpu().numpy(), np.where(np.arange(T * k) < n, order // k, -1))
    assert np.array_equal(got.offsets.cpu().numpy(), np.searchsorted(flat[order], np.arange(E + 1)))


@pytest.mark.parametrize("T,E,k,same", [(32768, 32, 2, True), (32768, 29, 3, False), (32769, 3, 1, True), (8192, 128, 4, False), (8177, 68, 5, True), (8193, 128, 4, False),
                                        (40000, 70, 2, False), (4099, 500, 7, False)])
def test_many_tokens(hero, T, E, k, same):
    """Counts added by the workgroups that place the rows, or by a scan, on either side of the choice; every token with the same experts: the largest sums."""
    l = _logits(T, E, "bf16", T + E)
    if same:
        l[:, E // 2] = 1000
    l[T // 2:T // 2 + 99] = -torch.inf
    got = hero.hero_moe_route(l.cuda(), k)
    v, i = l.float().sort(dim=1, descending=True, stable=True)
    flat = torch.where(v[:, :k] > -torch.inf, i[:, :k], E).reshape(-1).numpy()
    order = np.argsort(flat, kind="stable")
    n = int((flat < E).sum())
    slot = np.empty(T * k, np.int64)
    slot[order] = np.arange(T * k)
    assert np.array_equal(got.expert.cpu().numpy().reshape(-1), np.where(flat < E, flat, -1))
    assert np.array_equal(got.offsets.cpu().numpy(), np.searchsorted(flat[order], np.arange(E + 1)))
    assert np.array_equal(got.slot.cpu().numpy().reshape(-1), np.where(flat < E, slot, -1))
    assert np.array_equal(got.row_token.cpu().numpy(), np.where(np.arange(T * k) < n, order // k, -1))


def test_no_tokens(hero):
    got = hero.hero_moe_route(torch.empty((0, 6), device="cuda"), 2)
    assert got.offsets.tolist() == [0] * 7 and got.row_token.numel() == 0


@pytest.mark.parametrize("T", [40, 500])
def test_the_same_call_again_on_another_stream_and_replayed(hero, T):
    a, b = _logits(T, 64, "bf16", 1), _logits(T, 64, "bf16", 2)
    d, out = a.cuda(), hero.moe_routing(T, 64, 4)
    ws = torch.empty(hero.hero_moe_route_workspace_bytes(T, 64, 4), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    hero.hero_moe_route(d, 4, out=out, workspace=ws, stream=side)
    side.synchronize()
    _check(hero, a, 4, got=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hero.hero_moe_route(d, 4, out=out, workspace=ws)
    for x in (b, a, b):
        d.copy_(x)
        for t in out:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        _check(hero, x, 4, got=out)


def test_a_workspace_of_its_own_is_not_given_away_while_the_call_runs(hero):
    """The call makes its workspace and lets go of it before the stream has come to the kernels: what the current stream is then given is other memory."""
    T = 20000
    x = _logits(T, 64, "bf16", 3)
    d, out, side = x.cuda(), hero.moe_routing(T, 64, 4), torch.cuda.Stream()
    busy = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            busy = busy @ busy
    hero.hero_moe_route(d, 4, out=out, stream=side)
    need = hero.hero_moe_route_workspace_bytes(T, 64, 4)
    other = [torch.full((need,), 0x7f, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    _check(hero, x, 4, got=out)
    assert all((o == 0x7f).all() for o in other)


# ---------------------------------------------------------------------------------------- the weighted sum
def _combine_case(T, k, D, dt, seed, rows=None):
    g = torch.Generator().manual_seed(seed)
    n = T * k if rows is None else rows
    y, r = torch.randn((n, D), generator=g).to(TYPES[dt]), torch.randn((T, D), generator=g).to(TYPES[dt])
    slot = torch.randperm(T * k, generator=g).int().view(T, k)
    return y, slot, torch.rand((T, k), generator=g), r


def _check_combine(y, slot, weight, residual, got):
    f = lambda t: None if t is None else t.float().numpy()  # noqa: E731
    ref, mag = R.combine(f(y), slot.numpy(), weight.numpy(), f(residual))
    # fp32: each of the k products and additions and the residual's rounds once, 2^-24 of the sum of |terms| at most; then the result's type
    bound = R.EPS[y.dtype] * np.abs(ref) + (slot.shape[1] + 2) * 2.0 ** -24 * mag + 2.0 ** -25
    d = np.abs(got.cpu().double().numpy() - ref)
    assert (d <= bound).all(), np.max(d / bound)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("T,k,D", [(1, 1, 8), (1, 2, 768), (3, 8, 1032), (17, 3, 40), (100, 16, 256), (33, 4, 4096), (5, 6, 24)])
def test_weighted_sum(hero, T, k, D, dt):
    y, slot, w, r = _combine_case(T, k, D, dt, T + D)
    for res in (None, r):
        got = hero.hero_moe_combine(y.cuda(), slot.cuda(), w.cuda(), residual=None if res is None else res.cuda())
        _check_combine(y, slot, w, res, got)


def test_left_out_choices_whatever_lies_there(hero):
    y, slot, w, r = _combine_case(20, 3, 64, "bf16", 1)
    slot[3] = -1
    slot[4, 1], slot[5, 0], slot[6, 2] = -5, 60, 2 ** 31 - 1
    w[3], w[5, 0] = torch.inf, torch.nan
    unused = [x for x in range(60) if x not in slot.flatten().tolist()]
    y[unused] = torch.nan
    _check_combine(y, slot, w, r, hero.hero_moe_combine(y.cuda(), slot.cuda(), w.cuda(), residual=r.cuda()))
    got = hero.hero_moe_combine(y.cuda(), slot.cuda(), w.cuda())
    _check_combine(y, slot, w, None, got)
    assert (got[3] == 0).all()
    empty = hero.hero_moe_combine(torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), slot.cuda(), w.cuda(), residual=r.cuda())
    assert torch.equal(empty.cpu(), r)


def test_sum_in_place_into_wider_rows_and_the_same_row_twice(hero):
    y, slot, w, r = _combine_case(9, 2, 72, "f16", 2)
    slot[:, 1] = slot[:, 0]
    wide = torch.full((9, 88), 3.0, dtype=torch.float16, device="cuda")
    wide[:, 8:80] = r.cuda()
    yw = torch.zeros((18, 80), dtype=torch.float16, device="cuda")
    yw[:, :72] = y.cuda()
    stream = wide[:, 8:80]
    hero.hero_moe_combine(yw[:, :72], slot.cuda(), w.cuda(), residual=stream, out=stream)
    _check_combine(y, slot, w, r, stream)
    assert (wide[:, :8] == 3).all() and (wide[:, 80:] == 3).all()


def test_combine_rows_beyond_32_bits(hero):
    """Row offsets beyond 2^31 and 2^32 bytes."""
    D, n = 4096, 540_000                                                  # 4.4 GB
    y = torch.zeros((n, D), dtype=torch.bfloat16, device="cuda")
    picked = torch.tensor([[0, n - 1], [n - 2, 270_000], [262_144, 524_288], [300_000, 1]], dtype=torch.int32)
    for i, s in enumerate(picked.flatten().tolist()):
        y[s] = i + 1.0
    w = torch.tensor([[1.0, 0.5]] * 4)
    got = hero.hero_moe_combine(y, picked.cuda(), w.cuda()).cpu().float()
    assert torch.equal(got, torch.tensor([[1 + 1.0], [3 + 2.0], [5 + 3.0], [7 + 4.0]]).expand(4, D))
