"""The sparse prefill over a prompt read back from the cache, bit for bit against the prefill over the same numbers."""
import numpy as np
import pytest
import torch

import cache_oracle as co
import paper_2607_07724_amd as ugbs

from gpu_helpers import dev, dev_bf16
from test_gpu_cache import I32, PAGE, bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X (gfx950) visible to torch")
    ugbs.lib()


@pytest.mark.parametrize("backbone", [ugbs.KMEAN, ugbs.QUEST])
@pytest.mark.parametrize("d,dtype", [(64, ugbs.INT8), (128, ugbs.E4M3), (256, ugbs.E4M3)])
def test_prefill_over_a_cached_prompt_equals_the_prefill_over_its_numbers(d, dtype, backbone):
    g = np.random.default_rng(90 + d + backbone)
    B, H, Hkv, N = 2, 4, 2, 512
    c = ugbs.Cache.make(B, H, Hkv, d, 20, 8, rows=N, dtype=dtype)
    cbufs, step = ugbs.CacheBuffers(c), ugbs.CacheStep(c)
    step.plan(c, dev(np.array([N, N], I32)))
    given, expected = [], []
    for _ in range(2):
        bits, x = bf16(g.normal(0, 1, (B, Hkv, N, d)) * 2.0 ** g.integers(-3, 4, (B, Hkv, N, 1)))
        given.append(dev_bf16(bits))
        y = x.reshape(B, Hkv, N // PAGE, PAGE, d)
        s = np.vectorize(lambda a: co.scale_of(a, dtype))(np.abs(y).max((3, 4)))[..., None, None]
        back, value = bf16((co.nearest(y / s, dtype) * s).reshape(x.shape))
        assert np.array_equal(value, (co.nearest(y / s, dtype) * s).reshape(x.shape))      # (exact in bf16)
        expected.append(dev_bf16(back))
    ugbs.ugbs_cache_store(c, *given, step.slots, cbufs.cache, cbufs.scales)
    loaded = [torch.empty((B, Hkv, N, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    zero = torch.zeros(B, dtype=torch.int32, device="cuda")
    ugbs.ugbs_cache_load(c, cbufs.cache, cbufs.scales, step.table, zero, step.kv_lens, *loaded)
    p = ugbs.Problem.make(B, H, Hkv, N, d, 3, 0.25, backbone)
    Q = dev_bf16(bf16(g.normal(0, 1, (B, H, N, d)))[0])
    outs = []
    for K, V in (loaded, expected, given):
        O = torch.zeros((B, H, N, d), dtype=torch.bfloat16, device="cuda")
        ugbs.prefill(p, Q, K, V, O, ugbs.Buffers(p))
        outs.append(O.view(torch.int16))
    assert torch.equal(outs[0], outs[1])
    assert not torch.equal(outs[0], outs[2])             # (the rounding to 8 bits shows)
