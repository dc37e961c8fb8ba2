"""hero_layer_fwd_kv: a layer with 16-bit attention over a block-scaled 8-bit cache, prefill and decode, against the same layer put together
from the library's entry points, and against the layer that sees the whole sequence at once without a cache."""
import numpy as np
import pytest
import torch

import oracle as O
from oracle import layer as OL
from paper_2310_17723_amd import binding as HB
from paper_2310_17723_amd import synth
from parity import dev, upload_weights
from test_gpu_kv_cache import Pool

pytestmark = pytest.mark.gpu

MODES = {"M0": OL.MODE_M0, "M1": OL.MODE_M1, "mlp-block": OL.M_FC1 | OL.M_FC2}


def _layer(hero, arch, mode, hp, seed=51, **kw):
    base = dict(name="t", arch=arch, d=256, H=4, Dh=64, f=512, B=3, S=40, mask=synth.MASK_CAUSAL, eps=1e-5, w_std=0.04)
    base.update(kw)
    shape = synth.small(synth.CONFIGS[0], **base)
    odt, bit = (O.BF16, 0) if hp == "bf16" else (O.F16, HB.M_F16)
    p = synth.layer_params(seed, shape)
    hc = synth.activations(seed, shape, 2 * shape.B * shape.S, stream=1).astype(np.float64)
    sc, _ = OL.calibrate(p, hc, shape, 2 * shape.B, shape.S)
    W, t = upload_weights(hero, OL.prepare(p, sc, shape, MODES[mode], hp_dt=odt))
    desc = hero.layer_desc(shape.arch, shape.d, shape.H, shape.Dh, shape.f, shape.eps, shape.mask, MODES[mode] | bit)
    return shape, desc, W, t


def _by_hand(hero, shape, W, t, mode, h, cache, lens, new):
    """The pre-LN layer out of the entry points: LN^quant, QKV, write, attend, O (+h), LN^quant, FC1 + GELU, FC2 (+h)."""
    hp, (B, S, d, H, Dh) = h.dtype, (cache.sizes[0], h.shape[0] // cache.sizes[0], shape.d, shape.H, shape.Dh)
    mm = MODES[mode]
    yq, ys, yh = hero.hero_ln_quant(h, gamma=t["ln1_g"], beta=t["ln1_b"], eps=shape.eps, y_hp_dtype=hp)
    if mm & OL.M_QKV:
        qkv = hero.hero_int8_gemm(yq, t["w_qkv"], ys, t["w_qkv_s"], t["b_qkv"], epi=HB.EPI_DEQUANT, out_dtype=hp)
    else:
        qkv = hero.hero_hp_gemm(yh, t["w_qkv_hp"].view(hp), t["b_qkv"])
    q, k, v = (x.view(B, S, H, Dh) for x in qkv.view(B, S, 3 * d).split(d, 2))
    hero.hero_kv_write(cache, k, v, lens, new_len=new)
    a = hero.hero_kv_attn(cache, q, W.qk_scale, HB.MASK_CAUSAL, lens, new_len=new)
    h = hero.hero_hp_gemm(a, t["w_o_bf16"].view(hp), t["b_o"], residual=h)
    yq, ys, yh = hero.hero_ln_quant(h, gamma=t["ln2_g"], beta=t["ln2_b"], eps=shape.eps, y_hp_dtype=hp)
    if mm & OL.M_FC2:
        x = hero.hero_int8_gemm(yq, t["w_1"], ys, t["w_1_s"], t["b_1"], epi=HB.EPI_GELU_REQUANT, out_col_scale=t["S_a"], out_dtype=torch.int8)
        return hero.hero_int8_gemm(x, t["w_2"], None, t["w_2_s"], t["b_2"], residual=h, epi=HB.EPI_DEQUANT, out_dtype=hp)
    if mm & OL.M_FC1:
        x = hero.hero_int8_gemm(yq, t["w_1"], ys, t["w_1_s"], t["b_1"], epi=HB.EPI_DEQUANT_GELU, out_dtype=hp)
    else:
        x = hero.hero_hp_gemm(yh, t["w_1_hp"].view(hp), t["b_1"], gelu=True)
    return hero.hero_hp_gemm(x, t["w_2_bf16"].view(hp), t["b_2"], residual=h)


def _close(got, want, hp):
    """Two orders of the fp32 sums behind 16-bit roundings (QKV, attention, O, FC1, FC2 and the 8-bit codes between them, one of which may fall
    on the other side): the 16-bit class of a layer's outputs, 2e-2 of the larger of the value and the rms."""
    g, w = got.double(), want.double()
    rms = float(w.square().mean().sqrt())
    assert bool(((g - w).abs() <= 2e-2 * w.abs().clamp(min=rms)).all()), float(((g - w).abs() / w.abs().clamp(min=rms)).max())


@pytest.mark.parametrize("hp", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("mode", ["M0", "M1", "mlp-block"])
def test_pre_ln_prompt_then_tokens(hero, mode, fmt, hp):
    dt = torch.bfloat16 if hp == "bf16" else torch.float16
    shape, desc, W, t = _layer(hero, synth.PRE_LN, mode, hp)
    B, S, d = shape.B, shape.S, shape.d
    one, two = (Pool(hero, fmt, B, shape.H, shape.Dh, 16, 4, paged=True) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(3)
    lens, new = [S, S - 7, 3], [S, S - 7, 3]
    for step in range(4):
        n = S if step == 0 else (1 if step != 2 else 3)
        h = torch.randn((B * n, d), device="cuda", generator=g).to(dt)
        if step:
            lens, new = [x + n for x in lens], None
        ld, nd = torch.tensor(lens, dtype=torch.int32, device="cuda"), None if new is None else torch.tensor(new, dtype=torch.int32, device="cuda")
        want = _by_hand(hero, shape, W, t, mode, h.clone(), two.cache, ld, nd)
        ws = torch.empty(hero.hero_layer_kv_workspace_bytes(desc, one.cache, n), dtype=torch.uint8, device="cuda")
        hero.hero_layer_fwd_kv(desc, W, one.cache, n, ws, kv_len=ld, new_len=nd, h=h)
        rows = torch.arange(n, device="cuda")[None, :] < (torch.tensor(new, device="cuda")[:, None] if new else torch.full((B, 1), n, device="cuda"))
        _close(h[rows.view(-1)], want[rows.view(-1)], hp)
        a, b = hero.hero_kv_read(one.cache, 64, ld, dtype=torch.float32), hero.hero_kv_read(two.cache, 64, ld, dtype=torch.float32)
        for x, y in zip(a, b):
            for s in range(B):
                _close(x[s, :lens[s]], y[s, :lens[s]], hp)


@pytest.mark.parametrize("arch", [synth.PRE_LN, synth.POST_LN])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_tokens_one_by_one_are_the_whole_sequence(hero, fmt, arch):
    """A sequence through the cache, a prompt and then token by token, against the same layer over all of it at once without a cache.  The
    difference is K's and V's 8 bits: INT8 in blocks of 64 values a head wide is off by s / sqrt(12), s = absmax / 127 of some thousand values, i.e. about
    4 / 127 / 3.5 = 0.9 % of their rms; E4M3 by 2^-4 / sqrt(3) at most, 2.6 % on average.  The attention's output carries that and no more (an average of V,
    weights that differ by as much), and the layer's output a part of it: 3 % in norm."""
    shape, desc, W, t = _layer(hero, arch, "M1", "bf16", B=2, S=70)
    B, S, d = shape.B, shape.S, shape.d
    pool = Pool(hero, fmt, B, shape.H, shape.Dh, 64, 2)
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((B, S, d), device="cuda", generator=g).to(torch.bfloat16)

    def run(part, lens, cached):
        n = part.shape[1]
        rows = part.reshape(B * n, d).clone()                             # (the pre-LN layer updates its stream in place)
        ld = torch.tensor([lens] * B, dtype=torch.int32, device="cuda")
        kw = {}
        if arch == synth.POST_LN:
            q, s, _ = hero.hero_ln_quant(rows)
            kw = dict(x_q=q, x_scale=s, out_q=torch.empty((B * n, d), dtype=torch.int8, device="cuda"), out_scale=torch.empty(B * n, device="cuda"))
        else:
            kw = dict(h=rows)
        if cached:
            ws = torch.empty(hero.hero_layer_kv_workspace_bytes(desc, pool.cache, n), dtype=torch.uint8, device="cuda")
            hero.hero_layer_fwd_kv(desc, W, pool.cache, n, ws, kv_len=ld, **kw)
        else:
            ws = torch.empty(hero.hero_layer_workspace_bytes(desc, B, n), dtype=torch.uint8, device="cuda")
            hero.hero_layer_fwd(desc, W, B, n, ws, kv_len=ld, **kw)
        return (kw["out_q"].double() * kw["out_scale"].double()[:, None] if arch == synth.POST_LN else rows.double()).view(B, n, d)

    whole = run(x, S, False)
    parts = [run(x[:, :50], 50, True)] + [run(x[:, i:i + 1], i + 1, True) for i in range(50, S)]
    got = torch.cat(parts, 1)
    assert float((got - whole).norm() / whole.norm()) <= 3e-2


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_a_captured_step(hero, fmt):
    """A decode step captured once and replayed for other tokens and lengths in the same buffers, each replay against the step as it is called."""
    shape, desc, W, t = _layer(hero, synth.PRE_LN, "M1", "bf16")
    B, d = shape.B, shape.d
    one, two = (Pool(hero, fmt, B, shape.H, shape.Dh, 16, 4, paged=True) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(6)
    h, lens = torch.zeros((B, d), dtype=torch.bfloat16, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    ws, ws2 = (torch.empty(hero.hero_layer_kv_workspace_bytes(desc, one.cache, 1), dtype=torch.uint8, device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        hero.hero_layer_fwd_kv(desc, W, one.cache, 1, ws, kv_len=lens, h=h)      # (lengths of 0: nothing is written)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hero.hero_layer_fwd_kv(desc, W, one.cache, 1, ws, kv_len=lens, h=h)
    for step in range(20):
        x = torch.randn((B, d), device="cuda", generator=g).to(torch.bfloat16)
        h.copy_(x)
        lens.copy_(torch.tensor([step + 1, max(step - 3, 0), step + 1]))
        graph.replay()
        hero.hero_layer_fwd_kv(desc, W, two.cache, 1, ws2, kv_len=lens, h=x)
        assert torch.equal(h, x)
        torch.cuda.synchronize()
        for a, b in zip(hero.hero_kv_read(one.cache, 64, lens), hero.hero_kv_read(two.cache, 64, lens)):
            assert torch.equal(a, b)


def test_what_the_layer_refuses(hero):
    shape, desc, W, t = _layer(hero, synth.PRE_LN, "M1", "bf16")
    pool = Pool(hero, "i8", shape.B, shape.H, shape.Dh, 16, 4)
    ws = torch.empty(hero.hero_layer_kv_workspace_bytes(desc, pool.cache, 1), dtype=torch.uint8, device="cuda")
    h = torch.zeros((shape.B, shape.d), dtype=torch.bfloat16, device="cuda")
    lens = torch.ones(shape.B, dtype=torch.int32, device="cuda")

    def status(desc=desc, cache=pool.cache, S=1, h=h, lens=lens):
        try:
            hero.hero_layer_fwd_kv(desc, W, cache, S, ws, kv_len=lens, h=h)
        except HB.HeroError as e:
            return e.status
        return 0
    m2 = hero.layer_desc(shape.arch, shape.d, shape.H, shape.Dh, shape.f, shape.eps, shape.mask, HB.MODE_M2)
    assert status(desc=m2) == 4                                           # an INT8 attention has its own cache
    other = Pool(hero, "i8", shape.B, shape.H // 2, shape.Dh, 16, 4)
    assert status(cache=other.cache) == 2
    assert status(S=65) == 2                                              # more tokens than the cache holds
    assert status(lens=None) == 1 and status(h=None) == 1
    before = h.clone()
    assert torch.equal(h, before)
    assert status() == 0
