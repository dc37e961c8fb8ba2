"""The operators of a mixture-of-experts MLP together, as a pre-LN layer would run them: LN^quant, router, both linears, weighted sum."""
import numpy as np
import pytest
import torch

import moe_reference as R
import oracle as O
from paper_2310_17723_amd import binding as HB

pytestmark = pytest.mark.gpu


def _model(hero, E, d, f, fmt, seed):
    """Weights as the library prepares them (folded with the scale of the first linear's result), and their values."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    f8 = fmt == "e4m3"
    most = 448.0 if f8 else 127.0
    w1 = torch.randn((E, d, f), device="cuda", generator=g) / d ** 0.5
    w2 = torch.randn((E, f, d), device="cuda", generator=g) / f ** 0.5
    act = torch.rand((E, f), device="cuda", generator=g) * 0.5 / most + 3.5 / most
    q1 = [hero.hero_weight_fold_quant(w1[e], fp8=f8) for e in range(E)]
    q2 = [hero.hero_weight_fold_quant(w2[e], row_mult=act[e], fp8=f8) for e in range(E)]
    stack = lambda ts: torch.stack([t.view(torch.uint8) if t.element_size() == 1 else t for t in ts])  # noqa: E731
    c = torch.float8_e4m3fn if f8 else torch.int8
    return dict(w1=stack([q[0] for q in q1]).view(c), w1s=stack([q[1] for q in q1]), w2=stack([q[0] for q in q2]).view(c), w2s=stack([q[1] for q in q2]),
                b1=0.1 * torch.randn((E, f), device="cuda", generator=g), b2=0.1 * torch.randn((E, d), device="cuda", generator=g), act=act,
                router=(torch.randn((E, d), device="cuda", generator=g) * 2 / d ** 0.5).bfloat16())


def _mlp(hero, m, h, k, fmt, routing, ws, act, y):
    f8 = fmt == "e4m3"
    T, d = h.shape
    g, b = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")
    q, s, hp = hero.hero_ln_quant(h, gamma=g, beta=b, eps=1e-5, y_hp_dtype=torch.bfloat16, fp8=f8)
    E = m["router"].shape[0]
    logits = hero.hero_hp_gemm(hp, m["router"], C_out=torch.empty((T, E + -E % 4), dtype=hp.dtype, device="cuda")[:, :E])     # (rows of 8 bytes)
    product = hero.hero_fp8_gemm_grouped if f8 else hero.hero_int8_gemm_grouped
    r = hero.hero_moe_route(logits, k, out=routing, workspace=ws)
    product(q, m["w1"], r.offsets, row_index=r.row_token, a_row_scale=s, b_col_scale=m["w1s"], bias=m["b1"], epi=HB.EPI_GELU_REQUANT, out_col_scale=m["act"], C_out=act)
    product(act, m["w2"], r.offsets, b_col_scale=m["w2s"], bias=m["b2"], epi=HB.EPI_DEQUANT, C_out=y)
    hero.hero_moe_combine(y, r.slot, r.weight, residual=h, out=h)
    return q, s, logits


def _reference(m, h, q, s, logits, k, fmt):
    """64 bits on the CPU from the codes and logits that LN^quant and the router's product gave: (result, a bound of its error)."""
    x = q.float().cpu().double() * s.cpu().double()[:, None]
    expert, weight, *_ = R.route(logits.float().cpu().numpy(), k, True)
    out, slack = h.cpu().double(), torch.zeros(h.shape, dtype=torch.float64)
    mag = out.abs()
    half = 0.5 if fmt == "i8" else None
    for t in range(h.shape[0]):
        for j in range(k):
            e = int(expert[t, j])
            if e < 0:
                continue
            w1, w2 = (m[n][e].float().cpu().double() * m[n + "s"][e].cpu().double()[:, None] for n in ("w1", "w2"))
            a = R.gelu(x[t] @ w1.t() + m["b1"][e].cpu().double()) / m["act"][e].cpu().double()
            a = a.round().clamp(-127, 127) if fmt == "i8" else torch.from_numpy(O.e4m3_to_f32(O.f32_to_e4m3(a.clamp(-448, 448).float().numpy())).astype(np.float64))
            y = a @ w2.t() + m["b2"][e].cpu().double()
            out[t] += weight[t, j] * y
            mag[t] += abs(weight[t, j] * y)
            # a code that lies next to a border may be the neighbour: one step of up to four of the f codes (E4M3: the first product is off by a
            # little of its type's own, and one code in a hundred may be)
            steps = torch.full_like(a, 2 * half) if half else torch.exp2(torch.floor(torch.log2(a.abs().clamp(min=2.0 ** -6))) - 3)
            worst = (steps * w2.abs()).sort(dim=1, descending=True).values
            slack[t] += weight[t, j] * worst[:, :4 if fmt == "i8" else max(4, a.numel() // 100)].sum(1)
    return out, slack + 2 * 2.0 ** -8 * mag + 2.0 ** -16


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("T,E,k,d,f", [(1, 4, 2, 128, 256), (7, 8, 2, 256, 512), (90, 5, 3, 128, 384), (40, 70, 6, 128, 128)])
def test_all_of_it(hero, T, E, k, d, f, fmt):
    m = _model(hero, E, d, f, fmt, T)
    g = torch.Generator(device="cuda").manual_seed(T + 1)
    routing = hero.moe_routing(T, E, k)
    ws = torch.empty(hero.hero_moe_route_workspace_bytes(T, E, k), dtype=torch.uint8, device="cuda")
    act = torch.empty((T * k, f), dtype=m["w1"].dtype, device="cuda")
    y = torch.empty((T * k, d), dtype=torch.bfloat16, device="cuda")
    h0 = torch.randn((T, d), device="cuda", generator=g).bfloat16()
    h = h0.clone()
    q, s, logits = _mlp(hero, m, h, k, fmt, routing, ws, act, y)
    ref, bound = _reference(m, h0, q, s, logits, k, fmt)
    d_ = (h.cpu().double() - ref).abs()
    assert bool((d_ <= bound).all()), float((d_ / bound).max())

    # captured, and replayed on other rows with the program's own work in between
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                                         # (the first call of each kernel on the capture's stream is eager)
        _mlp(hero, m, h.clone(), k, fmt, routing, ws, act, y)
    torch.cuda.current_stream().wait_stream(side)
    hg = h0.clone()
    with torch.cuda.graph(graph):
        _mlp(hero, m, hg, k, fmt, routing, ws, act, y)
    for i in range(3):
        rows = torch.randn((T, d), device="cuda", generator=g).bfloat16()
        eager = rows.clone()
        _mlp(hero, m, eager, k, fmt, routing, ws, act, y)
        hg.copy_(rows)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(hg, eager)


def test_a_padding_token_keeps_its_row(hero):
    """Logits of -infinity: no expert, and the residual stream goes through unchanged."""
    m = _model(hero, 4, 128, 256, "i8", 3)
    h = torch.randn((6, 128), device="cuda").bfloat16()
    q, s, _ = hero.hero_ln_quant(h)
    logits = torch.randn((6, 4), device="cuda")
    logits[2], logits[5] = -torch.inf, -torch.inf
    r = hero.hero_moe_route(logits, 2)
    act = hero.hero_int8_gemm_grouped(q, m["w1"], r.offsets, row_index=r.row_token, a_row_scale=s, b_col_scale=m["w1s"], bias=m["b1"], epi=HB.EPI_GELU_REQUANT,
                                      out_col_scale=m["act"])
    y = hero.hero_int8_gemm_grouped(act, m["w2"], r.offsets, b_col_scale=m["w2s"], bias=m["b2"])
    out = hero.hero_moe_combine(y, r.slot, r.weight, residual=h)
    assert r.offsets[-1] == 8 and torch.equal(out[2], h[2]) and torch.equal(out[5], h[5]) and not torch.equal(out[0], h[0])
