"""The cache's calls without one of their tensors: a ValueError that names it, before the library is called."""
import pytest

import paper_2607_07724_amd as ugbs

torch = pytest.importorskip("torch")


class OnDevice:
    """What the binding asks of a device tensor, without a device."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, *shape, dtype=torch.int32):
        self.shape, self.dtype = torch.Size(shape), dtype

    def get_device(self):
        return 0

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x100000


def calls():
    c = ugbs.Cache.make(3, 8, 2, 128, 40, 10, rows=4)
    i32, bf = OnDevice, dict(dtype=torch.bfloat16)
    kv, q = OnDevice(3, 2, 4, 128, **bf), OnDevice(3, 8, 4, 128, **bf)
    cache, scales = OnDevice(40, 2, 2, 8192, dtype=torch.uint8), OnDevice(40, 2, 2, dtype=torch.float32)
    return c, {
        "ugbs_cache_plan": dict(ctx_lens=i32(3), new_lens=i32(3), free_pages=i32(40), free_count=i32(1), table=i32(3, 10),
                                kv_lens=i32(3), q_lens=i32(3), slots=i32(3, 4), free_left=i32(1)),
        "ugbs_cache_store": dict(K=kv, V=kv, slots=i32(3, 4), cache=cache, scales=scales),
        "ugbs_cache_load": dict(cache=cache, scales=scales, table=i32(3, 10), start=i32(3), count=i32(3), K=kv, V=kv),
        "ugbs_cache_attend": dict(Q=q, cache=cache, scales=scales, table=i32(3, 10), kv_lens=i32(3), q_lens=i32(3), O=q),
    }


@pytest.mark.parametrize("fn,name", [(fn, name) for fn, tensors in calls()[1].items() for name in tensors])
def test_a_missing_tensor_is_a_value_error(fn, name):
    c, tensors = calls()
    with pytest.raises(ValueError, match=name):
        getattr(ugbs, fn)(c, **{**tensors[fn], name: None})
