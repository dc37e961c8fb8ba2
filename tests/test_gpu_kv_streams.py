"""The block-scaled KV cache on another stream than the current one."""
import pytest
import torch

from test_gpu_kv_cache import Pool

pytestmark = pytest.mark.gpu


def test_rows_read_back_on_another_stream_while_the_current_one_is_busy(hero):
    """The outputs that the call makes are cleared before it writes them, whatever the current stream still has to do."""
    p = Pool(hero, "i8", 2, 3, 64, 16, 4, paged=True)
    lens = torch.tensor([64, 37], dtype=torch.int32, device="cuda")
    want = hero.hero_kv_read(p.cache, 64, lens, dtype=torch.float32)
    a = torch.ones((4096, 4096), device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):                                                   # (some ms)
        a = (a @ a) * 2.0 ** -12
    got = hero.hero_kv_read(p.cache, 64, lens, dtype=torch.float32, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and bool(want[0][0].any())
