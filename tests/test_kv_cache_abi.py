"""The block-scaled KV cache's entry points refuse what they cannot do before anything is launched (no GPU needed), and the structure that
describes a cache is laid out as the header says."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

from paper_2310_17723_amd import binding as HB

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4, 5
P = 0x10000                                                               # a placeholder address: nothing is dereferenced on these paths


@pytest.fixture(scope="module")
def lib():
    import paper_2310_17723_amd as pkg
    return pkg.load().lib


def _cache(**kw):
    d = dict(k=P, v=P, k_scale=P, v_scale=P, ks=(16 * 2 * 64, 64, 16 * 64, 1), vs=(16 * 2 * 64, 64, 16 * 64, 1), table=P, B=3, max_blocks=4,
             n_blocks=12, H=2, Dh=64, block=16, dt=HB.I8)
    d.update(kw)
    return HB.KvCache(d["k"], d["v"], d["k_scale"], d["v_scale"], (C.c_int64 * 4)(*d["ks"]), (C.c_int64 * 4)(*d["vs"]), d["table"], d["B"],
                      d["max_blocks"], d["n_blocks"], d["H"], d["Dh"], d["block"], d["dt"])


ST = (C.c_int64 * 4)(4 * 128, 128, 64, 1)


def _write(lib, c, k=P, v=P, ks=ST, vs=ST, dt=HB.BF16, S=4, kv_len=P, new_len=None):
    return lib.hero_kv_write(c, k, ks, v, vs, dt, S, kv_len, new_len, None)


def _read(lib, c, k=P, v=P, ks=ST, vs=ST, dt=HB.BF16, S=4, start=None, kv_len=P):
    return lib.hero_kv_read(c, k, ks, v, vs, dt, S, start, kv_len, None)


def _attn(lib, c, q=P, qs=ST, dt=HB.BF16, Hq=2, Sq=4, mask=HB.MASK_CAUSAL, kv_len=P, new_len=None, out=P, ldo=128, ws=None, nbytes=0):
    return lib.hero_kv_attn(c, q, qs, dt, Hq, Sq, 0.125, mask, kv_len, new_len, out, ldo, ws, nbytes, None)


BAD_CACHES = [(dict(Dh=96), UNSUPPORTED), (dict(Dh=256), UNSUPPORTED), (dict(block=8), UNSUPPORTED), (dict(block=48), UNSUPPORTED),
              (dict(block=256), UNSUPPORTED), (dict(block=0), UNSUPPORTED), (dict(dt=HB.U8), UNSUPPORTED), (dict(dt=HB.BF16), UNSUPPORTED),
              (dict(B=-1), SHAPE), (dict(H=-1), SHAPE), (dict(max_blocks=-1), SHAPE), (dict(n_blocks=-1), SHAPE), (dict(H=70000), SHAPE),
              (dict(max_blocks=2 ** 27), SHAPE), (dict(n_blocks=2 ** 31), SHAPE), (dict(table=None, n_blocks=11), SHAPE),
              (dict(k=None), NULL), (dict(v=None), NULL), (dict(k_scale=None), NULL), (dict(v_scale=None), NULL),
              (dict(ks=(2048, 64, 1024, 2)), UNSUPPORTED), (dict(vs=(2048, 72, 1024, 1)), ALIGN), (dict(ks=(2048, 64, 1000, 1)), ALIGN),
              (dict(ks=(2040, 64, 1024, 1)), ALIGN), (dict(vs=(-2048, 64, 1024, 1)), SHAPE), (dict(ks=(2048, -64, 1024, 1)), SHAPE),
              (dict(ks=(2048, 2 ** 28, 1024, 1)), SHAPE), (dict(block=128, vs=(4096, 2 ** 24, 1024, 1)), SHAPE), (dict(k=P + 8), ALIGN), (dict(v=P + 4), ALIGN), (dict(k_scale=P + 2), ALIGN),
              (dict(table=P + 1), ALIGN)]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_caches_that_are_refused(lib, kw, status):
    c = _cache(**kw)
    assert _write(lib, c) == status and _read(lib, c) == status and _attn(lib, c) == status
    assert lib.hero_kv_attn_workspace_bytes(c, 2, 1) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(dt=HB.F32), UNSUPPORTED), (dict(dt=HB.I8), UNSUPPORTED), (dict(S=-1), SHAPE), (dict(S=2 ** 31), SHAPE), (dict(k=None), NULL), (dict(v=None), NULL),
    (dict(ks=None), NULL), (dict(kv_len=None), NULL), (dict(kv_len=P + 2), ALIGN), (dict(new_len=P + 1), ALIGN), (dict(k=P + 2), ALIGN), (dict(v=P + 8), ALIGN),
    (dict(ks=(C.c_int64 * 4)(512, 128, 64, 2)), UNSUPPORTED), (dict(vs=(C.c_int64 * 4)(512, 124, 64, 1)), ALIGN), (dict(S=0), OK)])
def test_writes_that_are_refused(lib, kw, status):
    assert _write(lib, _cache(), **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dt=HB.I8), UNSUPPORTED), (dict(S=-1), SHAPE), (dict(k=None, v=None), NULL), (dict(vs=None), NULL), (dict(kv_len=None), NULL), (dict(start=P + 2), ALIGN),
    (dict(k=P + 8), ALIGN), (dict(k=None, ks=None, v=P + 8), ALIGN), (dict(vs=(C.c_int64 * 4)(512, 128, 60, 1)), ALIGN),
    (dict(ks=(C.c_int64 * 4)(512, 128, 64, 0)), UNSUPPORTED), (dict(S=0), OK)])
def test_reads_that_are_refused(lib, kw, status):
    assert _read(lib, _cache(), **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dt=HB.F32), UNSUPPORTED), (dict(mask=HB.MASK_PADDING), UNSUPPORTED), (dict(mask=7), UNSUPPORTED), (dict(Hq=3), SHAPE), (dict(Hq=-2), SHAPE),
    (dict(Sq=-1), SHAPE), (dict(Sq=2 ** 31), SHAPE), (dict(q=None), NULL), (dict(qs=None), NULL), (dict(out=None), NULL), (dict(kv_len=None), NULL),
    (dict(ldo=127), SHAPE), (dict(ldo=130), ALIGN), (dict(out=P + 8), ALIGN), (dict(q=P + 2), ALIGN), (dict(new_len=P + 3), ALIGN),
    (dict(qs=(C.c_int64 * 4)(512, 128, 64, 3)), UNSUPPORTED), (dict(qs=(C.c_int64 * 4)(512, 130, 64, 1)), ALIGN),
    (dict(ws=P + 128, nbytes=1 << 30), WORKSPACE), (dict(Sq=0), OK), (dict(Hq=0), OK)])
def test_attention_that_is_refused(lib, kw, status):
    assert _attn(lib, _cache(), **kw) == status


def test_a_kernel_that_is_not_there(lib):
    assert lib.hero_kv_attn_tile(_cache(), P, ST, HB.BF16, 2, 4, 0.125, HB.MASK_CAUSAL, P, None, P, 128, None, 0, None, 64) == UNSUPPORTED


def test_nothing_to_do(lib):
    for kw in (dict(B=0), dict(H=0)):
        c = _cache(k=None, v=None, k_scale=None, v_scale=None, **kw)
        assert _write(lib, c) == OK and _read(lib, c) == OK and _attn(lib, c, Hq=2 if c.H else 0) == OK
    assert lib.hero_kv_write(None, P, ST, P, ST, HB.BF16, 1, P, None, None) == NULL
    assert lib.hero_kv_attn_workspace_bytes(None, 2, 1) == 0
    assert lib.hero_kv_attn_workspace_bytes(_cache(), 3, 1) == 0


def test_workspace_of_few_rows_over_many_keys(lib):
    assert lib.hero_kv_attn_workspace_bytes(_cache(max_blocks=8192, n_blocks=1), 2, 1) > 0
    assert lib.hero_kv_attn_workspace_bytes(_cache(max_blocks=2, n_blocks=1), 2, 1) == 0


def test_the_structure_matches_the_header(tmp_path):
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "hero.h"', 'int main(void) {', '  printf("size %zu\\n", sizeof(hero_kv_cache));']
    lines += [f'  printf("{f} %zu\\n", offsetof(hero_kv_cache, {f}));' for f, _ in HB.KvCache._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ['  return 0;', '}']))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    seen = dict(line.split() for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    assert int(seen["size"]) == C.sizeof(HB.KvCache)
    for f, _ in HB.KvCache._fields_:
        assert int(seen[f]) == getattr(HB.KvCache, f).offset, f
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "hero.h")).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\}\s*hero_kv_cache;", text).group(1)
    assert sorted(re.findall(r"\b([A-Za-z_][A-Za-z0-9_]*)\s*(?:\[4\])?[;,]", body)) == sorted(f for f, _ in HB.KvCache._fields_)


def test_descriptions_that_are_refused():
    import paper_2310_17723_amd as pkg
    hero = pkg.load()
    k = torch.zeros((6, 16, 2, 64), dtype=torch.int8)
    s = torch.zeros((6, 2))
    c = hero.kv_cache(k, k.clone(), s, s.clone(), max_blocks=3, batch=2)
    assert (c.B, c.max_blocks, c.n_blocks, c.block, c.H, c.Dh, c.dt) == (2, 3, 6, 16, 2, 64, HB.I8) and list(c.k_strides) == list(k.stride())
    table = torch.zeros((2, 3), dtype=torch.int32)
    assert hero.kv_cache(k, k, s, s, block_table=table).max_blocks == 3
    for bad in (dict(k=k, v=k[:5], k_scale=s, v_scale=s, block_table=table), dict(k=k, v=k.float(), k_scale=s, v_scale=s, block_table=table),
                dict(k=k, v=k, k_scale=s.double(), v_scale=s, block_table=table), dict(k=k, v=k, k_scale=s, v_scale=s.t(), block_table=table),
                dict(k=k, v=k, k_scale=s, v_scale=s), dict(k=k, v=k, k_scale=s, v_scale=s, block_table=table.long()),
                dict(k=k, v=k, k_scale=s, v_scale=s, block_table=table, batch=5), dict(k=k, v=k, k_scale=s, v_scale=s, block_table=table.t())):
        with pytest.raises(ValueError):
            hero.kv_cache(**bad)
    with pytest.raises(ValueError):
        hero.kv_cache(k, k, s, s.to("meta"), block_table=table)
    with pytest.raises(AssertionError):
        hero.hero_kv_write(c, torch.zeros((2, 1, 3, 64), dtype=torch.bfloat16), torch.zeros((2, 1, 3, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(AssertionError):
        hero.hero_kv_attn(c, torch.zeros((2, 1, 2, 64), dtype=torch.bfloat16), 1.0, HB.MASK_CAUSAL, torch.zeros(2, dtype=torch.int64))


def test_layers_that_are_refused(lib):
    d = HB.LayerDesc(HB.ARCH_PRE_LN, 128, 2, 64, 256, 1e-5, HB.MASK_CAUSAL, HB.MODE_M1)
    w, io = HB.LayerWeights(), HB._LAYER_IO.pack(3, 1, 0, 0, 0, 0, P, P, 0, 0, 0, 0, 0, 0, 0)
    call = lambda d, io, c, new=None: lib.hero_layer_fwd_kv(d, w, io, c, new, C.c_void_p(P), 1 << 30, None)  # noqa: E731
    assert call(d, io, None) == NULL
    assert call(d, io, _cache(Dh=96)) == UNSUPPORTED and call(d, io, _cache(B=4)) == SHAPE and call(d, io, _cache(H=1)) == SHAPE
    assert call(HB.LayerDesc(HB.ARCH_PRE_LN, 128, 2, 64, 256, 1e-5, HB.MASK_CAUSAL, HB.MODE_M2), io, _cache()) == UNSUPPORTED
    assert call(d, HB._LAYER_IO.pack(3, 1, 0, 0, 0, 0, P, P, P, P, 64, 0, 0, 0, 0), _cache()) == UNSUPPORTED
    assert call(d, HB._LAYER_IO.pack(3, 65, 0, 0, 0, 0, P, P, 0, 0, 0, 0, 0, 0, 0), _cache()) == SHAPE
    assert call(d, HB._LAYER_IO.pack(3, 0, 0, 0, 0, 0, P, P, 0, 0, 0, 0, 0, 0, 0), _cache()) == OK
    assert lib.hero_layer_kv_workspace_bytes(d, _cache(), 1) > 0 and lib.hero_layer_kv_workspace_bytes(d, _cache(Dh=96), 1) == 0
    assert lib.hero_layer_kv_workspace_bytes(d, None, 1) == 0
    assert lib.hero_layer_kv_workspace_bytes(d, _cache(max_blocks=8192, n_blocks=1), 1) >= lib.hero_kv_attn_workspace_bytes(_cache(max_blocks=8192, n_blocks=1), 2, 1) > 0


def test_a_read_of_too_many_rows(lib):
    assert _read(lib, _cache(), S=1 << 30) == SHAPE


def test_more_threads_than_a_launch_has(lib):
    # 2^32 threads and more: 65535 x 300 rows of one workgroup each; 512 blocks of 65535 heads, one each; 2^29 rows of 8 threads
    assert _attn(lib, _cache(B=65535, H=300, n_blocks=1), Hq=300, Sq=1, ldo=300 * 64) == SHAPE
    assert _write(lib, _cache(H=65535, block=128, max_blocks=512, n_blocks=1), S=1 << 16) == SHAPE
    assert _read(lib, _cache(H=1 << 14, Dh=128), S=1 << 15) == SHAPE


@pytest.mark.parametrize("blocks", (dict(n_blocks=0), dict(max_blocks=0)))
def test_more_rows_than_fit_without_a_key(lib, blocks):
    c = _cache(B=65535, H=65535, **blocks)
    assert _attn(lib, c, Hq=65535, Sq=1 << 30, ldo=65535 * 64) == SHAPE     # (their elements pass 64 bits)


def test_a_cache_on_another_device_than_the_current_one(monkeypatch):
    import paper_2310_17723_amd as pkg
    hero = pkg.load()
    k, s = torch.zeros((6, 16, 2, 64), dtype=torch.int8), torch.zeros((6, 2))
    c = hero.kv_cache(k, k, s, s, max_blocks=3, batch=2)
    q, lens = torch.zeros((2, 1, 2, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in (lambda: hero.hero_kv_write(c, q, q, lens), lambda: hero.hero_kv_read(c, 1, lens), lambda: hero.hero_kv_attn(c, q, 1.0, HB.MASK_CAUSAL, lens)):
        with pytest.raises(ValueError):
            call()
    c.device = 1                                                          # rows that do not lie where the cache does
    with pytest.raises(AssertionError):
        hero.hero_kv_attn(c, q, 1.0, HB.MASK_CAUSAL, lens)


class _Elsewhere(torch.Tensor):
    def get_device(self):
        return 1


@pytest.mark.parametrize("part", ["out", "workspace"])
def test_a_result_or_a_workspace_on_another_device(part):
    import paper_2310_17723_amd as pkg
    hero, z = pkg.load(), lambda *s: torch.zeros(s, dtype=torch.int8)  # noqa: E731
    c = hero.kv_cache(z(4, 16, 2, 64), z(4, 16, 2, 64), torch.zeros(4, 2), torch.zeros(4, 2), max_blocks=2, batch=2)
    q, lens = torch.zeros((2, 1, 2, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    far = {"out": torch.zeros((2, 128), dtype=torch.bfloat16), "workspace": torch.zeros(256, dtype=torch.uint8)}[part].as_subclass(_Elsewhere)
    with pytest.raises(AssertionError, match=part if part == "workspace" else "result"):
        hero.hero_kv_attn(c, q, 1.0, HB.MASK_CAUSAL, lens, **{part: far})
