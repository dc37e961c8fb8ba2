"""The block-scaled KV cache, and what else clears its result itself, on another stream than the current one (no GPU needed: the library and the streams are stand-ins)."""
import contextlib
import types

import pytest
import torch

from paper_2310_17723_amd import binding as HB


@pytest.fixture
def hero(monkeypatch):
    """A binding whose library launches nothing; .on is the stream that torch's own kernels would go to, .log what was done and where."""
    h = object.__new__(HB.Hero)
    h.on, h.log = "current", []

    class Lib:
        def __getattr__(self, name):
            return lambda *args: h.log.append((name, args[-1])) or 0
    h.lib = Lib()

    @contextlib.contextmanager
    def stream(s):
        was, h.on = h.on, s.cuda_stream
        yield
        h.on = was
    monkeypatch.setattr(torch.cuda, "stream", stream)
    for where, name in ((torch, "zeros"), (torch.Tensor, "zero_")):
        monkeypatch.setattr(where, name, lambda *a, was=getattr(where, name), **k: h.log.append(("cleared", h.on)) or was(*a, **k))
    return h


class _Elsewhere(torch.Tensor):
    def get_device(self):
        return 1


def _cache(hero):
    z = lambda *s, dt=torch.int8: torch.empty(s, dtype=dt)  # noqa: E731
    return hero.kv_cache(z(4, 16, 2, 64), z(4, 16, 2, 64), z(4, 2, dt=torch.float32), z(4, 2, dt=torch.float32), max_blocks=2, batch=2)


def test_rows_read_back_are_cleared_on_the_stream_that_writes_them(hero):
    side = types.SimpleNamespace(cuda_stream="side", device_index=-1)
    out = torch.ones((2, 5, 2, 64), dtype=torch.bfloat16)
    for kw in (dict(), dict(v_out=out), dict(k_out=out)):
        hero.log.clear()
        k, v = hero.hero_kv_read(_cache(hero), 5, torch.empty(2, dtype=torch.int32), stream=side, **kw)
        assert [w for _, w in hero.log] == ["side"] * len(hero.log) and hero.log[-1][0] == "hero_kv_read" and len(hero.log) == 3 - len(kw)
        assert all(bool((t == 0).all()) or t is out for t in (k, v))


def test_column_maxima_are_cleared_on_the_stream_that_raises_them(hero):
    side = types.SimpleNamespace(cuda_stream="side", device_index=-1)
    hero.hero_absmax_cols(torch.ones((3, 8)), stream=side)
    assert [w for _, w in hero.log] == ["side", "side"]


def test_a_stream_of_another_device_than_the_cache(hero):
    """The kernels would run on the stream's device, without the cache's memory."""
    far = types.SimpleNamespace(cuda_stream="far", device_index=0)        # (the stand-in's tensors lie on the CPU, -1)
    c, lens = _cache(hero), torch.empty(2, dtype=torch.int32)
    q, ws = torch.empty((2, 1, 2, 64), dtype=torch.bfloat16), torch.empty(256, dtype=torch.uint8)
    desc, w = hero.layer_desc(HB.ARCH_PRE_LN, 128, 2, 64, 256, 1e-5, HB.MASK_CAUSAL, HB.MODE_M1), HB.LayerWeights()
    for call in (lambda: hero.hero_kv_write(c, q, q, lens, stream=far), lambda: hero.hero_kv_read(c, 1, lens, k_out=q, v_out=q, stream=far),
                 lambda: hero.hero_kv_attn(c, q, 1.0, HB.MASK_CAUSAL, lens, stream=far),
                 lambda: hero.hero_layer_fwd_kv(desc, w, c, 1, ws, kv_len=lens, stream=far)):
        with pytest.raises(ValueError, match="stream"):
            call()
    assert not hero.log


@pytest.mark.parametrize("name", ["x_q", "x_scale", "out_q", "out_scale", "h", "x_hp", "out_hp"])
def test_rows_of_another_number_or_device_than_the_cache_has(hero, name):
    """The kernels would read and write batch * S rows, the batch being the cache's, whatever the tensors hold."""
    stream = types.SimpleNamespace(cuda_stream="side", device_index=-1)
    c, lens, ws = _cache(hero), torch.empty(2, dtype=torch.int32), torch.empty(256, dtype=torch.uint8)
    desc, w = hero.layer_desc(HB.ARCH_PRE_LN, 128, 2, 64, 256, 1e-5, HB.MASK_CAUSAL, HB.MODE_M1), HB.LayerWeights()
    size = lambda n: (n,) if name.endswith("scale") else (n, 128)  # noqa: E731
    for bad in (torch.empty(size(3)), torch.empty(size(7))):
        with pytest.raises(HB.HeroError, match="rows") as e:
            hero.hero_layer_fwd_kv(desc, w, c, 3, ws, kv_len=lens, stream=stream, **{name: bad})
        assert e.value.status == 2
    with pytest.raises(AssertionError, match="rows"):
        hero.hero_layer_fwd_kv(desc, w, c, 3, ws, kv_len=lens, stream=stream, **{name: torch.empty(size(6)).as_subclass(_Elsewhere)})
    assert not hero.log
    hero.hero_layer_fwd_kv(desc, w, c, 3, ws, kv_len=lens, stream=stream, **{name: torch.empty(size(6))})
    assert hero.log == [("hero_layer_fwd_kv", "side")]
