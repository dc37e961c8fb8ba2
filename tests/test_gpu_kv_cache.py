"""The block-scaled 8-bit KV cache, hero_kv_write and hero_kv_read: every byte of the pool and every scale against a plain
implementation (tests/kv_reference.py), bit for bit; what no call names stays as it was."""
import numpy as np
import pytest
import torch

import kv_reference as R

pytestmark = pytest.mark.gpu
HP = {"bf16": torch.bfloat16, "f16": torch.float16}


class Pool:
    """A cache on the GPU and its twin on the CPU.  layout: "heads" [n, H, block, Dh], "tokens" [n, block, H, Dh], "fused" K and V
    side by side in one buffer of tokens, with rows that are longer than they need to be."""

    def __init__(self, hero, fmt, B, H, Dh, block, max_blocks, paged=False, layout="heads", seed=0, fill=None, extra=2):
        self.hero, self.fmt, self.block, self.H, self.Dh, self.B = hero, fmt, block, H, Dh, B
        g = np.random.default_rng(seed)
        n = B * max_blocks + extra
        self.table = (g.permutation(n)[:B * max_blocks] if paged else np.arange(B * max_blocks)).reshape(B, max_blocks).astype(np.int32)
        limit = 256 if fmt == "i8" else 127                               # (no NaN among the codes that lie there before)
        self.codes = {x: g.integers(0, limit, (n, H, block, Dh)).astype(np.uint8) if fill is None else np.full((n, H, block, Dh), fill, np.uint8) for x in "kv"}
        self.scale = {x: g.uniform(0.001, 0.02, (n, H)).astype(np.float32) for x in "kv"}
        shape = {"heads": (n, H, block, Dh), "tokens": (n, block, H, Dh)}.get(layout)
        if layout == "fused":
            buf = torch.full((n, block, 2 * H, Dh + 16), 77, dtype=torch.uint8, device="cuda")
            self.raw = {"k": buf[:, :, :H, :Dh], "v": buf[:, :, H:, :Dh]}
            self.buf = buf
        else:
            self.raw = {x: torch.empty(shape, dtype=torch.uint8, device="cuda") for x in "kv"}
            if layout == "heads":
                self.raw = {x: t.transpose(1, 2) for x, t in self.raw.items()}
        for x in "kv":                                                    # [n, block, H, Dh] views
            self.raw[x].copy_(torch.from_numpy(self.codes[x]).cuda().transpose(1, 2))
        self.dev_scale = {x: torch.from_numpy(self.scale[x].copy()).cuda() for x in "kv"}
        self.dev_table = torch.from_numpy(self.table).cuda() if paged else None
        dt = R.FORMATS[fmt][0]
        self.cache = hero.kv_cache(self.raw["k"].view(dt), self.raw["v"].view(dt), self.dev_scale["k"], self.dev_scale["v"],
                                   max_blocks=max_blocks, batch=B, block_table=self.dev_table)

    def write(self, k, v, kv_len, new_len=None, **kw):
        dev = lambda a: None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
        self.hero.hero_kv_write(self.cache, k, v, dev(kv_len), new_len=dev(new_len), **kw)
        for x, t in (("k", k), ("v", v)):
            R.write(self.codes[x], self.scale[x], self.table, t.float().cpu().numpy(), kv_len, new_len, self.fmt)

    def check(self):
        torch.cuda.synchronize()
        for x in "kv":
            s = self.dev_scale[x].cpu().numpy()
            assert np.array_equal(s, self.scale[x], equal_nan=True), (x, np.flatnonzero(s != self.scale[x])[:5])
            c = self.raw[x].transpose(1, 2).contiguous().cpu().numpy()
            z = self.fmt == "e4m3"                                        # (+0 and -0 are the same value)
            bad = (c != self.codes[x]) & ~(z & ((c & 127) == 0) & ((self.codes[x] & 127) == 0))
            assert not bad.any(), (x, np.argwhere(bad)[:5], c[bad][:5], self.codes[x][bad][:5])


def _rows(seed, B, S, H, Dh, dt, spread=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((B, S, H, Dh), device="cuda", generator=g)
    if spread:                                                            # tokens of very different size: scales grow within a block
        x = x * torch.exp2(torch.randint(-6, 7, (B, S, 1, 1), device="cuda", generator=g).float())
    return x.to(dt)


@pytest.mark.parametrize("layout", ["heads", "tokens", "fused"])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("Dh,H,block", [(64, 3, 16), (128, 2, 32), (64, 1, 64), (128, 5, 128)])
@pytest.mark.parametrize("hp", ["bf16", "f16"])
def test_rows_of_any_number_at_any_position(hero, hp, Dh, H, block, fmt, layout):
    mb = 4
    for S in (1, 5, block, block + 3, 2 * block + 7):
        p = Pool(hero, fmt, 4, H, Dh, block, mb, paged=S % 2 == 1, layout=layout, seed=S)
        p.write(_rows(S, 4, S, H, Dh, HP[hp]), _rows(S + 1, 4, S, H, Dh, HP[hp]), [S, S + 3, min(mb * block, S + block - 1), mb * block])
        p.check()
    if layout == "fused":
        assert bool((p.buf[..., Dh:] == 77).all())


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("block", [16, 64])
def test_token_by_token(hero, block, fmt):
    """A cache filled one token at a time: the scale of a block grows as its tokens do, its older ones are coded anew."""
    p = Pool(hero, fmt, 2, 3, 64, block, 3, paged=True)
    for t in range(2 * block + 3):
        p.write(_rows(t, 2, 1, 3, 64, torch.bfloat16), _rows(t + 1000, 2, 1, 3, 64, torch.bfloat16), [t + 1, t + 2])
        if t % 7 == 0 or t > 2 * block:
            p.check()
    p.check()


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_a_padded_batch_and_lengths_out_of_range(hero, fmt):
    """new_len of 0, beyond S and negative; lengths that begin before position 0, end behind the last block, are 0 or negative."""
    B, S, H, Dh, block, mb = 9, 11, 2, 64, 16, 2
    p = Pool(hero, fmt, B, H, Dh, block, mb)
    k, v = _rows(1, B, S, H, Dh, torch.float16), _rows(2, B, S, H, Dh, torch.float16)
    new = [0, 3, 11, 40, -5, 7, 7, 11, 1]
    k[1, 3:] = float("nan")                                               # rows that hold no token are not looked at
    v[5, 7:] = float("inf")
    p.write(k, v, [20, 5, 4, 30, 9, 0, -3, 40, 33], new)
    p.check()
    q = Pool(hero, fmt, B, H, Dh, block, mb, paged=True)
    q.write(k.nan_to_num(), v.nan_to_num(0, 1, 1), [2 ** 31 - 1, 2 ** 31 - 6, 3, 11, 12, 32, 35, 43, -2 ** 31])
    q.check()


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_an_index_that_is_no_block(hero, fmt):
    B, S, H, Dh, block, mb = 3, 40, 2, 128, 16, 4
    p = Pool(hero, fmt, B, H, Dh, block, mb, paged=True)
    p.table[0, 1], p.table[1, 0], p.table[2, 2] = -1, 10 ** 9, p.codes["k"].shape[0]
    p.dev_table.copy_(torch.from_numpy(p.table))
    p.write(_rows(3, B, S, H, Dh, torch.bfloat16), _rows(4, B, S, H, Dh, torch.bfloat16), [40, 50, 60])
    p.check()
    lens = torch.tensor([40, 50, 60], dtype=torch.int32, device="cuda")
    ko, vo = hero.hero_kv_read(p.cache, 64, lens, dtype=torch.float32)
    for x, o in (("k", ko), ("v", vo)):
        for b in range(B):
            ref, _ = R.rows_of(p.codes[x], p.scale[x], p.table, b, int(lens[b]), fmt)
            assert np.array_equal(o[b, :lens[b]].cpu().numpy(), ref.astype(np.float32)) and not bool(o[b, lens[b]:].any())


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("hp", ["bf16", "f16"])
def test_values_of_all_sizes(hero, hp, fmt):
    """Rows of zeros, of the type's smallest and largest numbers, and next to ties of the codes."""
    B, S, H, Dh, block = 8, 16, 2, 64, 16
    big = torch.finfo(HP[hp]).max
    x = _rows(5, B, S, H, Dh, HP[hp], spread=False)
    x[0] = 0
    x[1] = x[1].sign() * torch.finfo(HP[hp]).smallest_normal / 2
    x[2] = x[2].sign() * big
    x[3] = (x[3].float().clamp(-0.9, 0.9) * big).to(HP[hp])
    x[4] = (torch.randint(-254, 255, x[4].shape, device="cuda") / 2).to(HP[hp])                   # halves of whole numbers, the largest 127
    x[4, ..., 0] = 127
    x[5] = (torch.randint(-31, 32, x[5].shape, device="cuda") * 16).clamp(-448, 448).to(HP[hp])   # and of the E4M3 grid
    x[5, ..., 0] = 448
    x[6] = (x[6].float() * 1e-7).to(HP[hp])
    p = Pool(hero, fmt, B, H, Dh, block, 2)
    p.write(x, x.flip(3), [S] * B)
    p.check()
    p.write((x * 3).nan_to_num(0, big, -big)[:, :5], x[:, :5], [S + 5] * B)
    p.check()


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_is_no_number_is_not_silent(hero, bad, fmt):
    """The block and head that hold it read as NaN, the others do not; begun anew, the block is clean again."""
    B, S, H, Dh, block = 2, 20, 3, 64, 16
    p = Pool(hero, fmt, B, H, Dh, block, 2)
    k, v = _rows(6, B, S, H, Dh, torch.bfloat16), _rows(7, B, S, H, Dh, torch.bfloat16)
    p.write(k, v, [S] * B)
    p.check()
    k1 = _rows(8, B, 1, H, Dh, torch.bfloat16)
    k1[1, 0, 2, 17] = bad
    p.write(k1, v[:, :1], [S + 1] * B)
    p.check()
    lens = torch.tensor([S + 1] * B, dtype=torch.int32, device="cuda")
    ko, vo = hero.hero_kv_read(p.cache, S + 1, lens)
    want = torch.zeros(ko.shape, dtype=torch.bool, device="cuda")
    want[1, 16:, 2] = True
    assert torch.equal(torch.isnan(ko), want) and not bool(torch.isnan(vo).any())
    p.write(v[:, :1], v[:, :1], [S + 2] * B)                              # still so
    p.check()
    p.write(k, v, [S] * B)                                                # begun anew
    p.check()
    assert not bool(torch.isnan(hero.hero_kv_read(p.cache, S, lens)[0]).any())


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("Dh,block,layout", [(64, 16, "tokens"), (128, 64, "heads"), (128, 32, "fused")])
def test_reading_back(hero, Dh, block, layout, dt, fmt):
    """Any window of any sequence, into strided outputs whose other rows keep what they hold."""
    B, H, mb, S = 5, 3, 3, block + 9
    p = Pool(hero, fmt, B, H, Dh, block, mb, paged=True, layout=layout)
    lens, start = [0, 1, block + 5, 3 * block, 4 * block], [0, 0, 3, 2 * block - 2, -4]
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    buf = torch.full((2, B, H, S + 1, Dh + 8), 7.5, dtype=dt, device="cuda")
    ko, vo = (t[:, :, :S, :Dh].transpose(1, 2) for t in buf)
    hero.hero_kv_read(p.cache, S, dev(lens), start=dev(start), k_out=ko, v_out=vo)
    for x, o in (("k", ko), ("v", vo)):
        want = torch.full((B, S, H, Dh), 7.5, dtype=torch.float64)
        for b in range(B):
            ref, _ = R.rows_of(p.codes[x], p.scale[x], p.table, b, min(lens[b], mb * block), fmt)
            for i in range(S):
                if 0 <= start[b] + i < len(ref):
                    want[b, i] = torch.from_numpy(ref[start[b] + i])
        # code * scale is rounded to fp32 (2^-24), then to the type (half a step, at most eps / 2 of the value; FP16 below its normal numbers 2^-25)
        tol = want.abs() * (torch.finfo(dt).eps / 2 * (dt != torch.float32) + 2.0 ** -23) + (2.0 ** -25 if dt == torch.float16 else 0)
        assert bool(((o.double().cpu() - want).abs() <= tol).all())
    assert bool((buf[..., Dh:] == 7.5).all()) and bool((buf[:, :, :, S:] == 7.5).all())


def test_a_captured_write_and_read(hero):
    """A step captured into a graph and replayed with other tokens in the same buffers, eager work between the replays."""
    B, H, Dh, block = 3, 4, 128, 16
    p = Pool(hero, "i8", B, H, Dh, block, 4)
    k, v = (torch.zeros((B, 1, H, Dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    ko, vo = (torch.zeros((B, 64, H, Dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        hero.hero_kv_write(p.cache, k, v, lens)                           # (lengths of 0: nothing is written)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hero.hero_kv_write(p.cache, k, v, lens)
        hero.hero_kv_read(p.cache, 64, lens, k_out=ko, v_out=vo)
    p.check()
    for t in range(20):
        k.copy_(_rows(t, B, 1, H, Dh, torch.bfloat16))
        v.copy_(_rows(t + 50, B, 1, H, Dh, torch.bfloat16))
        lens.copy_(torch.tensor([t + 1, t + 5, t + 16]))
        graph.replay()
        for x, n in (("k", k), ("v", v)):
            R.write(p.codes[x], p.scale[x], p.table, n.float().cpu().numpy(), [t + 1, t + 5, t + 16], None, "i8")
        p.check()
        a, b = hero.hero_kv_read(p.cache, 64, lens)
        for got, want in ((ko, a), (vo, b)):
            for s in range(B):
                assert torch.equal(got[s, :lens[s]], want[s, :lens[s]])
