"""hero_kv_attn, 16-bit attention over the block-scaled 8-bit cache, against 64 bits on the same codes and scales."""
import numpy as np
import pytest
import torch

import kv_reference as R
from paper_2310_17723_amd import binding as HB
from test_gpu_kv_cache import HP, Pool, _rows

pytestmark = pytest.mark.gpu


def _dev(a):
    return None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")


TILES = [None, 16, 32, 256]                                               # the library's choice of a kernel, and each kernel


def _attend(p, q, scale, mask, lens, new=None, workspace=True, **kw):
    ws = None
    if workspace:
        n = p.hero.hero_kv_attn_workspace_bytes(p.cache, q.shape[2], q.shape[1]) if kw.get("tile") is None else 64 << 20
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    return p.hero.hero_kv_attn(p.cache, q, scale, mask, _dev(lens), new_len=_dev(new), workspace=ws, **kw)


def _check(p, q, scale, mask, lens, new=None, got=None, **kw):
    y = (_attend(p, q, scale, mask, lens, new, **kw) if got is None else got).double().cpu().numpy().reshape(q.shape)
    half = 2.0 ** -8 if q.dtype == torch.bfloat16 else 2.0 ** -11         # half a step of the result's type, relative
    B, S, Hq, Dh = q.shape
    cap = p.table.shape[1] * p.block
    for b in range(B):
        L, n = min(max(lens[b], 0), cap), S if new is None else min(max(new[b], 0), S)
        (ks, _), (vs, v_scale) = (R.rows_of(p.codes[x], p.scale[x], p.table, b, L, p.fmt) for x in "kv")
        ref, mag, size, peak = R.attend(q[b].double().cpu().numpy(), ks, vs, v_scale, scale, mask == HB.MASK_CAUSAL, n)
        # P is rounded to FP16 (2^-11), numerator and denominator: twice; the scores' fp32 sums are off by Dh 2^-24 of sum |q k| at most,
        # the addend log2(vs) and the maximum by a few 2^-24 of values below 2^7, and so are the exponentials, twice; below 2^-29 of the largest P
        # is a subnormal number, off by 2^-40 of the largest (p times V's scale) for each key and step of its code
        slack = 2 * (Dh + 8) * 2.0 ** -24 * size + 2.0 ** -15
        bound = (2 * 2.0 ** -11 + slack) * mag + 2.0 ** -39 * R.FORMATS[p.fmt][1] * peak + half * np.abs(ref) + 2.0 ** -25
        bad = ~(np.abs(y[b] - ref) <= bound)
        assert not bad.any(), (b, np.argwhere(bad)[:4], y[b][bad][:4], ref[bad][:4], np.max(np.abs(y[b] - ref) / bound))


def _filled(hero, fmt, B, H, Dh, block, mb, seed=0, **kw):
    """A pool whose blocks were written; what lies behind the lengths are bytes of all kinds, E4M3's NaN among them."""
    p = Pool(hero, fmt, B, H, Dh, block, mb, seed=seed, fill=0x7f, **kw)
    return p


def _fill(p, lens, seed, dt):
    S = max(max(lens), 1)
    k, v = _rows(seed, p.B, S, p.H, p.Dh, dt, spread=False), _rows(seed + 1, p.B, S, p.H, p.Dh, dt)
    cap = p.table.shape[1] * p.block
    n = [min(max(x, 0), cap) for x in lens]
    p.write(k[:, :max(n)], v[:, :max(n)], n, n)


@pytest.mark.parametrize("hp", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("Dh,block,layout", [(64, 16, "tokens"), (128, 64, "heads"), (128, 16, "fused"), (64, 128, "heads")])
@pytest.mark.parametrize("H,group", [(3, 1), (2, 4), (1, 7)])
def test_one_token(hero, H, group, Dh, block, layout, fmt, hp):
    """Generation: lengths around the steps of keys and the ends of blocks, empty and overlong ones among them."""
    lens = [0, 1, 15, 16, 17, 31, 32, 33, 100, 129, 255, 256, 257, 300, -3]
    p = _filled(hero, fmt, len(lens), H, Dh, block, -(-256 // block), paged=True, layout=layout)
    _fill(p, lens, 11, HP[hp])
    q = _rows(12, len(lens), 1, H * group, Dh, HP[hp], spread=False)
    for mask in (HB.MASK_NONE, HB.MASK_CAUSAL):
        _check(p, q, Dh ** -0.5, mask, lens)


@pytest.mark.parametrize("hp", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("mask", [HB.MASK_NONE, HB.MASK_CAUSAL])
@pytest.mark.parametrize("S,H,group,Dh", [(2, 2, 1, 64), (5, 1, 4, 128), (16, 2, 1, 128), (9, 1, 7, 64), (31, 1, 2, 128), (33, 2, 1, 64),
                                          (70, 1, 1, 128), (50, 1, 3, 64), (130, 2, 1, 64), (150, 1, 2, 128), (260, 1, 1, 128)])
def test_several_tokens(hero, S, H, group, Dh, mask, fmt, hp):
    """Drafted tokens, chunks and whole prompts in a padded batch: keys before the call or none, rows that hold no token, rows that see no key
    (a length below the number of new tokens)."""
    lens, new = [S, S + 1, S + 37, S + 90, max(1, S // 2), 0, S + 64], [S, S, S, max(1, S - 1), S, 0, max(1, S // 3)]
    p = _filled(hero, fmt, len(lens), H, Dh, 32, (S + 96) // 32 + 1, paged=True)
    _fill(p, lens, S, HP[hp])
    q = _rows(13, len(lens), S, H * group, Dh, HP[hp], spread=False)
    _check(p, q, Dh ** -0.5, mask, lens, new)
    _check(p, q, Dh ** -0.5, mask, lens)
    for tile in TILES[1:]:
        _check(p, q, Dh ** -0.5, mask, lens, new, tile=tile)


@pytest.mark.parametrize("hp", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("Dh,block,layout", [(64, 16, "tokens"), (128, 64, "heads"), (128, 16, "fused"), (64, 128, "heads"), (64, 64, "fused"), (128, 32, "tokens"), (128, 128, "heads")])
@pytest.mark.parametrize("S,group", [(1, 1), (20, 4), (300, 1)])
def test_every_kernel_on_every_layout(hero, S, group, Dh, block, layout, fmt, hp):
    H, lens = 2, [S, S + 1, S + 63, S + 129]
    p = _filled(hero, fmt, len(lens), H, Dh, block, -(-(S + 129) // block), paged=True, layout=layout)
    _fill(p, lens, S + Dh, HP[hp])
    q = _rows(14, len(lens), S, H * group, Dh, HP[hp], spread=False)
    for tile in TILES[1:]:
        for mask in (HB.MASK_NONE, HB.MASK_CAUSAL):
            _check(p, q, Dh ** -0.5, mask, lens, tile=tile)


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("S,group,B", [(1, 1, 1), (1, 8, 2), (3, 4, 1), (40, 1, 1), (200, 1, 1)])
def test_keys_in_pieces(hero, S, group, B, fmt):
    """Few rows over many keys are split along the keys; without a workspace they are not."""
    H, Dh, block, L = 2, 128, 64, 5000
    lens = [L, 700][:B]
    p = _filled(hero, fmt, B, H, Dh, block, -(-L // block), paged=True)
    _fill(p, lens, 21, torch.bfloat16)
    q = _rows(22, B, S, H * group, Dh, torch.bfloat16, spread=False)
    assert hero.hero_kv_attn_workspace_bytes(p.cache, H * group, S) > 0
    one, two = _attend(p, q, Dh ** -0.5, HB.MASK_CAUSAL, lens), _attend(p, q, Dh ** -0.5, HB.MASK_CAUSAL, lens)
    assert torch.equal(one, two)                                          # the order of the sums is fixed
    _check(p, q, Dh ** -0.5, HB.MASK_CAUSAL, lens, got=one)
    _check(p, q, Dh ** -0.5, HB.MASK_CAUSAL, lens, workspace=False)
    for tile in TILES[1:]:
        _check(p, q, Dh ** -0.5, HB.MASK_CAUSAL, lens, tile=tile)
        _check(p, q, Dh ** -0.5, HB.MASK_CAUSAL, lens, tile=tile, workspace=False)


@pytest.mark.parametrize("S", [1, 40, 140])
@pytest.mark.parametrize("scale", [-0.125, 0.0, 1e-30, 0.7])
@pytest.mark.parametrize("hp", ["bf16", "f16"])
def test_scales_and_sizes_of_queries(hero, hp, scale, S):
    """Any scale; rows of queries from the type's smallest numbers to large ones, of zeros, and with one value far above the others."""
    H, Dh = 8, 64
    p = _filled(hero, "i8", 2, H, Dh, 64, 4)
    lens = [200, 256]
    _fill(p, lens, 31, HP[hp])
    q = _rows(32, 2, S, H, Dh, torch.float32, spread=False)
    size = [1e-38, 1e-20, 0.0, 1.0, 300.0, 1e-4, 1.0, 7.0] if hp == "bf16" else [6e-8, 1e-5, 0.0, 1.0, 300.0, 1e-4, 1.0, 7.0]
    q = q * torch.tensor(size, device="cuda")[:, None]
    q[:, :, 6, 3] = 3e4
    for tile in TILES:
        _check(p, q.to(HP[hp]), scale if scale != 0.7 else 0.7 / 300, HB.MASK_CAUSAL, lens, tile=tile)


@pytest.mark.parametrize("S", [1, 20, 140])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_blocks_of_very_different_size(hero, fmt, S):
    """V of 2^-20 .. 2^20 from block to block (its scale enters through the exponent), a block of zeros with most of the weight, and a
    long flat tail of small probabilities."""
    H, Dh, block, L = 2, 64, 16, 480
    p = _filled(hero, fmt, 3, H, Dh, block, L // block)
    k, v = _rows(41, 3, L, H, Dh, torch.bfloat16, spread=False), _rows(42, 3, L, H, Dh, torch.bfloat16, spread=False)
    q = _rows(43, 3, S, H, Dh, torch.bfloat16, spread=False)
    v[0] = (v[0].float() * torch.exp2((torch.arange(L, device="cuda") // block % 9 * 5 - 20).float())[:, None, None]).to(torch.bfloat16)
    v[1, 32:48] = 0
    k[1, :, :, 0], q[1, :, :, 0] = 0, 4
    k[1, 32:48, :, 0] = 40                                                # (score 160 / 8 above the others)
    k[2], q[2] = 0, 0
    k[2, 77, :, 0], q[2, :, :, 0] = 16, 8                                 # e^16 times as likely as each of the others
    v[2, 77] = 0
    p.write(k, v, [L] * 3)
    for tile in TILES:
        _check(p, q, Dh ** -0.5, HB.MASK_NONE, [L] * 3, tile=tile)


@pytest.mark.parametrize("S,group", [(1, 1), (4, 4), (64, 3)])
def test_an_index_that_is_no_block(hero, S, group):
    """Its keys are left out; a sequence without any block outputs 0."""
    H, Dh, block = 2, 128, 16
    p = _filled(hero, "e4m3", 4, H, Dh, block, 8, paged=True)
    lens = [128, 100, 90, 128]
    _fill(p, lens, 51, torch.float16)
    p.table[0, 1], p.table[1, 0], p.table[1, 6], p.table[2, 4], p.table[3] = -1, 10 ** 9, -7, p.codes["k"].shape[0], -1
    p.dev_table.copy_(torch.from_numpy(p.table))
    for tile in TILES:
        _check(p, _rows(52, 4, S, H * group, Dh, torch.float16, spread=False), 0.1, HB.MASK_CAUSAL, lens, tile=tile)


@pytest.mark.parametrize("S,group", [(1, 1), (20, 1), (40, 4), (140, 2)])
def test_a_scale_that_is_no_number_reaches_who_sees_it(hero, S, group):
    """A NaN among the tokens of a block: rows that see a key of that block and head are NaN, all others as without it."""
    H, Dh, block = 3, 64, 16
    p = _filled(hero, "i8", 2, H, Dh, block, -(-(S + 60) // block) + 1)
    lens = [S + 60, S + 60]
    k, v = (_rows(s, 2, S + 60, H, Dh, torch.bfloat16, spread=False) for s in (61, 62))
    at = S + 58                                                           # the last rows alone see its block
    k[0, at, 1, 5], v[1, at, 2, 7] = float("nan"), float("inf")
    p.write(k, v, lens)
    q = _rows(63, 2, S, H * group, Dh, torch.bfloat16, spread=False)
    ys = [_attend(p, q, 0.1, HB.MASK_CAUSAL, lens, tile=tile).view(2, S, H, group, Dh) for tile in TILES]
    first = at // block * block - 60                                      # the first row that sees the block
    want = torch.zeros((2, S, H, group, Dh), dtype=torch.bool, device="cuda")
    want[0, max(first, 0):, 1], want[1, max(first, 0):, 2] = True, True
    for x in "kv":                                                        # the same without the blocks that are NaN
        p.scale[x] = np.nan_to_num(p.scale[x], nan=1.0)
        p.dev_scale[x].copy_(torch.from_numpy(p.scale[x]))
    for tile, y in zip(TILES, ys):
        assert torch.equal(torch.isnan(y), want)
        z = _attend(p, q, 0.1, HB.MASK_CAUSAL, lens, tile=tile).view_as(y)
        assert torch.equal(y[~want], z[~want])


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("hp", ["bf16", "f16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_query_that_is_no_number_stays_in_its_row(hero, bad, hp, tile):
    H, group, Dh, S = 2, 2, 64, 50
    p = _filled(hero, "e4m3", 2, H, Dh, 16, 8)
    _fill(p, [120, 77], 91, HP[hp])
    q = _rows(92, 2, S, H * group, Dh, HP[hp], spread=False)
    y = _attend(p, q, 0.1, HB.MASK_CAUSAL, [120, 77], tile=tile).view(2, S, H * group, Dh)
    q[1, 17, 3, 5] = bad
    z = _attend(p, q, 0.1, HB.MASK_CAUSAL, [120, 77], tile=tile).view_as(y)
    rest = torch.ones((2, S, H * group), dtype=torch.bool, device="cuda")
    rest[1, 17, 3] = False
    assert bool(torch.isnan(z[1, 17, 3]).all()) and torch.equal(z[rest], y[rest])


@pytest.mark.parametrize("tile", TILES)
def test_scores_that_rise_and_a_score_beyond_fp32(hero, tile):
    """The maximum rises in every step of keys, by little, by more than FP16 holds, from far below; and a row whose score fp32 does not
    hold is NaN, not zeros."""
    H, Dh, S, L = 1, 64, 40, 320
    p = _filled(hero, "i8", 4, H, Dh, 16, L // 16)
    k, v, q = (torch.zeros((4, n, H, Dh), device="cuda") for n in (L, L, S))
    v[:] = _rows(95, 4, L, H, Dh, torch.float32, spread=False)
    at = torch.arange(L, device="cuda").float()
    k[0, :, 0, 0], k[1, :, 0, 0], k[2, :, 0, 0] = at / 10, at * 2, at / 4 - 400
    k[3, :, 0, 0] = 1e30
    q[:, :, 0, 0] = 1.0
    q[3, 17, 0, 0] = 1e10
    for x in (k, v):
        x.copy_(x.to(torch.bfloat16))
    p.write(k.to(torch.bfloat16), v.to(torch.bfloat16), [L] * 4)
    y = _attend(p, q.to(torch.bfloat16), 1.0, HB.MASK_NONE, [L] * 4, tile=tile).view(4, S, Dh)
    assert bool(torch.isnan(y[3, 17]).all()) and not bool(torch.isnan(y[:3]).any())
    three = Pool(hero, "i8", 3, H, Dh, 16, L // 16, fill=0x7f)
    three.write(k[:3].to(torch.bfloat16), v[:3].to(torch.bfloat16), [L] * 3)
    _check(three, q[:3].to(torch.bfloat16), 1.0, HB.MASK_NONE, [L] * 3, tile=tile)


@pytest.mark.parametrize("S", [1, 40, 140])
def test_strides_and_rows_of_the_output(hero, S):
    """Queries out of a fused buffer, an output with a leading dimension of its own: what lies between its rows stays."""
    H, group, Dh, lens = 2, 2, 64, [S + 50, S + 9]
    p = _filled(hero, "i8", 2, H, Dh, 32, -(-(S + 50) // 32))
    _fill(p, lens, 71, torch.bfloat16)
    buf = _rows(72, 2, S, H * group * 3 + 1, Dh, torch.bfloat16, spread=False)
    q = buf[:, :, 1:1 + H * group]
    for tile in TILES:
        out = torch.full((2 * S, H * group * Dh + 12), 7.0, dtype=torch.bfloat16, device="cuda")
        _attend(p, q, 0.125, HB.MASK_CAUSAL, lens, out=out[:, :H * group * Dh], tile=tile)
        assert bool((out[:, H * group * Dh:] == 7.0).all())
        _check(p, q, 0.125, HB.MASK_CAUSAL, lens, got=out[:, :H * group * Dh].contiguous())


def test_a_cache_without_blocks(hero):
    codes, scale = torch.zeros((0, 16, 2, 64), dtype=torch.int8, device="cuda"), torch.zeros((0, 2), device="cuda")
    table = torch.zeros((3, 4), dtype=torch.int32, device="cuda")
    c = hero.kv_cache(codes, codes, scale, scale, block_table=table)
    lens = torch.tensor([5, 0, 9], dtype=torch.int32, device="cuda")
    q = _rows(1, 3, 2, 4, 64, torch.float16)
    hero.hero_kv_write(c, q[:, :, :2], q[:, :, :2], lens)
    assert not bool(hero.hero_kv_attn(c, q, 1.0, HB.MASK_CAUSAL, lens).any())
    assert not bool(hero.hero_kv_read(c, 9, lens)[0].any())


def test_many_rows_without_a_block(hero):
    """More than 2^23 values to clear, rows apart from each other."""
    B, S, H = 2, 9001, 8
    codes = torch.empty((0, 16, H, 64), dtype=torch.int8, device="cuda")
    scales = torch.empty((0, H), device="cuda")
    cache = hero.kv_cache(codes, codes, scales, scales, max_blocks=0, batch=B)
    q = torch.ones((B, S, H, 64), dtype=torch.bfloat16, device="cuda")
    buf = torch.full((B * S, H * 64 + 12), 7.0, dtype=torch.bfloat16, device="cuda")
    hero.hero_kv_attn(cache, q, 0.1, HB.MASK_NONE, _dev([0, 5]), out=buf[:, :H * 64])
    assert int(buf[:, :H * 64].count_nonzero()) == 0 and bool((buf[:, H * 64:] == 7.0).all())


FAR = {"blocks": (2 ** 30, 256, 128, 2 ** 29), "rows": (4096, 2 ** 24 - 16, 128, 2 ** 23), "heads": (2 ** 20, 128, 2 ** 32, 2 ** 31)}    # block, token (as far as it may), head, V behind K


@pytest.mark.parametrize("far", sorted(FAR))
def test_offsets_that_pass_32_bits(hero, far):
    """Blocks, tokens of a block or heads that lie so far apart that their offsets pass 31 or 32 bits: the bits of the same cache in one piece."""
    B, H, Dh, block, mb = 2, 2, 128, 128, 2
    near = _filled(hero, "i8", B, H, Dh, block, mb, paged=True)
    lens = [135, 256]
    _fill(near, lens, 5, torch.bfloat16)
    n = near.raw["k"].shape[0]
    sb, sr, sh, sv = FAR[far]
    buf = torch.empty((n - 1) * sb + (block - 1) * sr + (H - 1) * sh + sv + Dh, dtype=torch.int8, device="cuda")
    k, v = (buf[off:].as_strided((n, block, H, Dh), (sb, sr, sh, 1), off) for off in (0, sv))
    k.copy_(near.raw["k"].view(torch.int8))
    v.copy_(near.raw["v"].view(torch.int8))
    scales = [near.dev_scale[x].clone() for x in "kv"]
    cache = hero.kv_cache(k, v, *scales, block_table=near.dev_table)
    lens = [136, 256]
    kn, vn = _rows(7, B, 1, H, Dh, torch.bfloat16), _rows(8, B, 1, H, Dh, torch.bfloat16)
    near.write(kn, vn, lens)
    hero.hero_kv_write(cache, kn, vn, _dev(lens))
    near.check()
    assert all(torch.equal(s, near.dev_scale[x]) for s, x in zip(scales, "kv"))
    for x, y in zip(hero.hero_kv_read(cache, 256, _dev(lens)), hero.hero_kv_read(near.cache, 256, _dev(lens))):
        assert torch.equal(x, y)
    for S, tile in ((1, 16), (9, 32), (70, 256)):
        q = _rows(9, B, S, 2 * H, Dh, torch.bfloat16, spread=False)
        got = hero.hero_kv_attn(cache, q, 0.088, HB.MASK_CAUSAL, _dev(lens), tile=tile)
        assert torch.equal(got, hero.hero_kv_attn(near.cache, q, 0.088, HB.MASK_CAUSAL, _dev(lens), tile=tile))
        _check(near, q, 0.088, HB.MASK_CAUSAL, lens, got=got)


@pytest.mark.parametrize("S,tile", [(20, 16), (20, 32), (33, 256)])
def test_rows_that_lie_far_apart(hero, S, tile):
    """Queries, rows to write, rows read and results whose offsets pass 32 bits: tokens 2^27 values apart."""
    B, H, Dh, block, step = 2, 2, 64, 32, 2 ** 27
    p, lens = _filled(hero, "i8", B, H, Dh, block, 3), [S, 96]
    buf = torch.empty(B * S * step, dtype=torch.bfloat16, device="cuda")
    place = lambda i, heads: buf.as_strided((B, S, heads, Dh), (S * step, step, Dh, 1), i * 1024)  # noqa: E731
    k, v, q, ko, vo = (place(i, h) for i, h in enumerate((H, H, 2 * H, H, H)))
    for x, seed in ((k, 1), (v, 2), (q, 3)):
        x.copy_(_rows(seed, B, S, x.shape[2], Dh, torch.bfloat16, spread=False))
    _fill(p, [96, 96], 5, torch.bfloat16)
    p.write(k, v, lens)
    p.check()
    start = _dev([x - S for x in lens])
    hero.hero_kv_read(p.cache, S, _dev(lens), start=start, k_out=ko, v_out=vo)
    for x, y in zip(hero.hero_kv_read(p.cache, S, _dev(lens), start=start), (ko, vo)):
        assert torch.equal(x, y)
    out = buf.as_strided((B * S, 2 * H * Dh), (step, 1), 8192)
    hero.hero_kv_attn(p.cache, q, 0.125, HB.MASK_CAUSAL, _dev(lens), out=out, tile=tile)
    _check(p, q, 0.125, HB.MASK_CAUSAL, lens, got=out.contiguous())


@pytest.mark.parametrize("hp", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_a_prompt_then_tokens(hero, fmt, hp):
    """As they are used together: prompts of different lengths written and attended over, then generation, then drafted tokens, some of
    which are taken back and written over, on a stream of its own and with a graph of the step."""
    B, H, group, Dh, block = 3, 2, 4, 128, 16
    p = _filled(hero, fmt, B, H, Dh, block, 8, paged=True)
    dt, lens = HP[hp], [37, 5, 64]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        S = 64
        k, v, q = _rows(81, B, S, H, Dh, dt, False), _rows(82, B, S, H, Dh, dt), _rows(83, B, S, H * group, Dh, dt, False)
        p.write(k, v, lens, lens)
        _check(p, q, Dh ** -0.5, HB.MASK_CAUSAL, lens, lens)
        for t in range(6):
            S = 1 if t != 3 else 5
            if t == 4:
                lens = [x - 3 for x in lens]                              # drafted tokens taken back
            lens = [x + S for x in lens]
            k, v, q = _rows(90 + t, B, S, H, Dh, dt, False), _rows(190 + t, B, S, H, Dh, dt), _rows(290 + t, B, S, H * group, Dh, dt, False)
            p.write(k, v, lens)
            _check(p, q, Dh ** -0.5, HB.MASK_CAUSAL, lens)
        p.check()
        # the step as a graph
        kg, vg, qg, lg = k.clone(), v.clone(), q.clone(), _dev(lens)
        ws = torch.empty(hero.hero_kv_attn_workspace_bytes(p.cache, H * group, 1), dtype=torch.uint8, device="cuda")
        out = torch.empty((B, H * group * Dh), dtype=dt, device="cuda")
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hero.hero_kv_write(p.cache, kg, vg, lg)
        hero.hero_kv_attn(p.cache, qg, Dh ** -0.5, HB.MASK_CAUSAL, lg, out=out, workspace=ws)
    for t in range(5):
        lens = [x + 1 for x in lens]
        for buf, seed in ((kg, 400), (vg, 500), (qg, 600)):
            buf.copy_(_rows(seed + t, B, 1, buf.shape[2], Dh, dt, False))
        lg.copy_(_dev(lens))
        graph.replay()
        for x, n in (("k", kg), ("v", vg)):
            R.write(p.codes[x], p.scale[x], p.table, n.float().cpu().numpy(), lens, None, fmt)
        p.check()
        _check(p, qg, Dh ** -0.5, HB.MASK_CAUSAL, lens, got=out)
        assert torch.equal(out, _attend(p, qg, Dh ** -0.5, HB.MASK_CAUSAL, lens))
