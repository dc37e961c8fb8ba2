"""hero_layer_fwd_kv's attention module alone: the MLP's second linear is zero and the attention-output linear eight times as large, so that a layer's output is what
its attention found in the cache (beside the residual stream).  The rows are compared with 64 bits on the layer's own cache, and the same reference with one key
less, or without the last piece of the keys, has to lie outside the tolerance."""
import numpy as np
import pytest
import torch

import kv_reference as R
from oracle import layer as OL
from paper_2310_17723_amd import binding as HB
from paper_2310_17723_amd import synth
from test_gpu_kv_cache import HP, Pool
from test_gpu_kv_layer import MODES, _layer

pytestmark = pytest.mark.gpu


def _attention_alone(hero, arch, mode, hp, **kw):
    shape, desc, W, t = _layer(hero, arch, mode, hp, **kw)
    w = t["w_o_bf16"].view(HP[hp])
    w.mul_(8)                                                             # (a power of two: exact)
    for name in ("w_2_bf16", "b_2", "b_o"):
        t[name].zero_()
    return shape, desc, W, t


def _qkv(hero, shape, t, mode, x, hp):
    """This call's q, k, v [B, n, H, Dh] out of the entry points.  x: the pre-LN stream, or the post-LN layer's codes and scales."""
    if isinstance(x, tuple):
        yq, ys, yh = *x, None
    else:
        yq, ys, yh = hero.hero_ln_quant(x, gamma=t["ln1_g"], beta=t["ln1_b"], eps=shape.eps, y_hp_dtype=x.dtype)
    if MODES[mode] & OL.M_QKV:
        y = hero.hero_int8_gemm(yq, t["w_qkv"], ys, t["w_qkv_s"], t["b_qkv"], epi=HB.EPI_DEQUANT, out_dtype=HP[hp])
    else:
        y = hero.hero_hp_gemm(yh, t["w_qkv_hp"].view(HP[hp]), t["b_qkv"])
    return [z.view(shape.B, -1, shape.H, shape.Dh).double().cpu().numpy() for z in y.split(shape.d, 1)]


def _from_the_gpu(p):
    for x in "kv":
        p.codes[x] = p.raw[x].transpose(1, 2).contiguous().cpu().numpy()
        p.scale[x] = p.dev_scale[x].cpu().numpy()


def _attend(p, q, b, L, n, W, cut=0):
    """The rows of sequence b: (attention W_o^T, a bound for it) with its last `cut` keys left out.  q and k come out of 16-bit roundings that another order of sums may
    take the other way (half a step of size = sum |q k|), P and the attention's result are rounded too; W_o's product carries that in norm."""
    (ks, _), (vs, v_scale) = (R.rows_of(p.codes[x], p.scale[x], p.table, b, L - cut, p.fmt) for x in "kv")
    a, mag, size, _ = R.attend(q[b], ks, vs, v_scale, q.shape[3] ** -0.5, True, n)
    eps = 2.0 ** -8 if W.dtype == torch.bfloat16 else 2.0 ** -11
    w = W.double().cpu().numpy()
    err = eps * np.abs(a) + (2.0 ** -10 + 2.0 ** -15 + 2 * eps * size) * mag
    S = a.shape[0]
    return a.reshape(S, -1) @ w.T, np.linalg.norm(err.reshape(S, -1), axis=1) * np.linalg.norm(w, 2)


def _ln(x, g, b, eps):
    return (x - x.mean(1, keepdims=True)) / np.sqrt(x.var(1, keepdims=True) + eps) * g + b


def _step(hero, shape, desc, W, t, mode, hp, pool, g, lens, new, n, cut=1):
    """One call of n tokens (new of them in a padded batch), its rows against the reference."""
    B, d, post, dt = shape.B, shape.d, shape.arch == synth.POST_LN, HP[hp]
    dev = lambda a: None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    h = (torch.randn((B * n, d), device="cuda", generator=g) / 16).to(dt)
    kw = dict(h=h.clone())
    if post:
        xq, xs, _ = hero.hero_ln_quant(h)
        kw = dict(x_q=xq, x_scale=xs, out_q=torch.empty((B * n, d), dtype=torch.int8, device="cuda"), out_scale=torch.empty(B * n, device="cuda"))
    q, k, v = _qkv(hero, shape, t, mode, (xq, xs) if post else h, hp)
    ws = torch.empty(hero.hero_layer_kv_workspace_bytes(desc, pool.cache, n), dtype=torch.uint8, device="cuda")
    hero.hero_layer_fwd_kv(desc, W, pool.cache, n, ws, kv_len=dev(lens), new_len=dev(new), **kw)
    torch.cuda.synchronize()
    _from_the_gpu(pool)
    eps, Wo = (2.0 ** -8 if hp == "bf16" else 2.0 ** -11), t["w_o_bf16"].view(dt)
    for b in range(B):
        m = n if new is None else new[b]
        for x, rows in (("k", k), ("v", v)):                              # the new tokens lie where they belong: off by half a code and a 16-bit rounding
            got, scale = R.rows_of(pool.codes[x], pool.scale[x], pool.table, b, lens[b], pool.fmt)
            got, scale, want = got[lens[b] - m:], scale[lens[b] - m:, :, None], rows[b, :m]
            # (a later token of the call may have raised the scale: this call's rows are coded once all the same)
            tol = (scale / 2 if pool.fmt == "i8" else np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * scale)) * 1.001 + 2 * eps * np.abs(want)
            assert (np.abs(got - want) <= tol).all(), (x, b)
        (o, bound), (o1, _) = (_attend(pool, q, b, lens[b], m, Wo, c) for c in (0, cut))
        rows = slice(b * n, b * n + m)
        if post:
            x0 = xq[rows].double().cpu().numpy() * xs[rows].double().cpu().numpy()[:, None]
            p = {key: t[key].double().cpu().numpy() for key in ("ln1_g", "ln1_b", "ln2_g", "ln2_b")}
            want, wrong = (_ln(_ln(x0 + y[:m], p["ln1_g"], p["ln1_b"], shape.eps), p["ln2_g"], p["ln2_b"], shape.eps) for y in (o, o1))
            got, s = kw["out_q"][rows].double().cpu().numpy(), kw["out_scale"][rows].double().cpu().numpy()
            # the sum's error through two layer norms (their gains over its deviation), X_o's 16 bits, and half a code of X_mid's rows and of the result's, d values each
            sd = (x0 + o[:m]).std(1)
            gain = np.abs(p["ln1_g"]).max() * np.abs(p["ln2_g"]).max() / sd
            mid = _ln(x0 + o[:m], p["ln1_g"], p["ln1_b"], shape.eps)
            tol = 1.1 * (gain * (bound[:m] + eps * np.linalg.norm(o[:m], axis=1)) + d ** 0.5 / 2 / 127 * np.abs(mid).max(1) * np.abs(p["ln2_g"]).max() / mid.std(1) + d ** 0.5 / 2 * s)
            got = got * s[:, None]
        else:
            x0 = h[rows].double().cpu().numpy()
            want, wrong, got = x0 + o[:m], x0 + o1[:m], kw["h"][rows].double().cpu().numpy()
            tol = bound[:m] + (2 * eps + 2.0 ** -16) * np.linalg.norm(want, axis=1)      # (the stream is rounded behind O, and behind FC2 once more)
        off, planted = np.linalg.norm(got - want, axis=1), np.linalg.norm(wrong - want, axis=1)
        assert (off <= tol).all(), (b, off / tol)
        assert (planted > tol).any(), (b, planted / tol)                  # a layer that left those keys out (off = planted) would not pass


@pytest.mark.parametrize("hp", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("arch,mode", [(synth.PRE_LN, "M0"), (synth.PRE_LN, "M1"), (synth.POST_LN, "M1")])
def test_what_attention_finds_in_the_cache(hero, arch, mode, fmt, hp):
    """A padded prompt, tokens one by one, drafted ones: one key less would be seen."""
    shape, desc, W, t = _attention_alone(hero, arch, mode, hp)
    pool = Pool(hero, fmt, shape.B, shape.H, shape.Dh, 16, 4, paged=True)
    g = torch.Generator(device="cuda").manual_seed(5)
    lens = [6, 9, 3]
    _step(hero, shape, desc, W, t, mode, hp, pool, g, lens, lens, 9)
    for n in (1, 1, 3, 1, 2, 1):
        lens = [x + n for x in lens]
        _step(hero, shape, desc, W, t, mode, hp, pool, g, lens, None, n)


@pytest.mark.parametrize("hp", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("arch", [synth.PRE_LN, synth.POST_LN])
def test_a_step_whose_keys_are_split(hero, arch, fmt, hp):
    """Behind some 2000 keys the attention's pieces lie in the scratch that the linears share.  V is positive but for every other channel of the last 512 keys: a row
    without that piece would have those channels twice as large (a layer norm behind it sees that, too)."""
    shape, desc, W, t = _attention_alone(hero, arch, "M1", hp, B=2)
    pool = Pool(hero, fmt, shape.B, shape.H, shape.Dh, 64, 32, paged=True, seed=3)
    r, dt = np.random.default_rng(9), R.FORMATS[fmt][0]
    k, v = r.uniform(-120, 120, pool.codes["k"].shape), r.uniform(30, 120, pool.codes["v"].shape)
    v[pool.table[:, 24:].reshape(-1), ..., ::2] *= -1
    for x, values in (("k", k), ("v", v)):
        pool.codes[x] = torch.from_numpy(values).to(dt).view(torch.uint8).numpy()
        pool.raw[x].copy_(torch.from_numpy(pool.codes[x]).cuda().transpose(1, 2))
        pool.scale[x] = r.uniform(0.009, 0.011, pool.scale[x].shape).astype(np.float32)
        pool.dev_scale[x].copy_(torch.from_numpy(pool.scale[x]))
    assert hero.hero_kv_attn_workspace_bytes(pool.cache, shape.H, 1) > 0 and hero.hero_kv_attn_workspace_bytes(pool.cache, shape.H, 3) > 0
    g = torch.Generator(device="cuda").manual_seed(6)
    for lens, n in (([2000, 1900], 1), ([2003, 1903], 3), ([2048, 1904], 1)):
        _step(hero, shape, desc, W, t, "M1", hp, pool, g, lens, None, n, cut=512)


def test_a_refused_call_touches_nothing(hero):
    """The residual stream, which a layer updates in place, and the cache are what they were before."""
    shape, desc, W, t = _layer(hero, synth.PRE_LN, "M1", "bf16")
    pool, other = Pool(hero, "i8", shape.B, shape.H, shape.Dh, 16, 4), Pool(hero, "i8", shape.B, shape.H // 2, shape.Dh, 16, 4)
    h = torch.randn((shape.B * 65, shape.d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).to(torch.bfloat16)
    before, lens = h.clone(), torch.ones(shape.B, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(hero.hero_layer_kv_workspace_bytes(desc, pool.cache, n) for n in (1, 65)), dtype=torch.uint8, device="cuda")
    make = lambda mask, mode: hero.layer_desc(shape.arch, shape.d, shape.H, shape.Dh, shape.f, shape.eps, mask, mode)  # noqa: E731
    for kw, status in ((dict(desc=make(shape.mask, HB.MODE_M2)), 4), (dict(desc=make(7, HB.MODE_M1)), 4), (dict(cache=other.cache), 2), (dict(n=65), 2), (dict(lens=None), 1),
                       (dict(ws=ws[:256]), 5)):
        n = kw.get("n", 1)
        with pytest.raises(HB.HeroError) as e:
            hero.hero_layer_fwd_kv(kw.get("desc", desc), W, kw.get("cache", pool.cache), n, kw.get("ws", ws), kv_len=kw.get("lens", lens), h=h[:shape.B * n])
        assert e.value.status == status, kw
    torch.cuda.synchronize()
    assert torch.equal(h, before)
    pool.check()
    other.check()
    hero.hero_layer_fwd_kv(desc, W, pool.cache, 1, ws, kv_len=lens, h=h[:shape.B])
    assert not torch.equal(h[:shape.B], before[:shape.B]) and torch.equal(h[shape.B:], before[shape.B:])
