"""What a chunk and a paged cache keep of the tensors and bounds that they were made from (host tensors that pass
for device ones: nothing is launched)."""
import ctypes

import pytest
import torch

import paper_2501_13111_amd as fp
from paper_2501_13111_amd.paged import _Chunk


class Dev(torch.Tensor):
    is_cuda = True


def dev(t):
    return torch.Tensor._make_subclass(Dev, t)


def cache(page=64, dtype=torch.bfloat16):
    sc = [dev(torch.zeros(10, 2, page, dtype=torch.float16)) for _ in range(2)] if dtype == torch.int8 else []
    return fp.PagedKV(dev(torch.zeros(10, 2, page, 64, dtype=dtype)), dev(torch.zeros(10, 2, page // 32, 64, 32, dtype=dtype)), *sc)


def chunk(**kw):
    return fp.Chunk(dev(torch.zeros(4, dtype=torch.int32)), dev(torch.zeros(3, dtype=torch.int32)),
                    dev(torch.zeros(3, 5, dtype=torch.int32)), **dict(dict(max_new=4), **kw))


def struct(c, kv, n):
    return ctypes.cast(c.c(kv, n), ctypes.POINTER(_Chunk)).contents


def test_a_chunk_does_not_change_under_its_calls():
    c, kv = chunk(max_len=200), cache()
    before = struct(c, kv, 7)
    assert (before.max_new, before.max_len, before.ctx_len) == (4, 200, c.ctx_len.data_ptr())
    for name, value in (("max_new", 9), ("max_len", 100), ("ctx_len", c.ctx_len + 1), ("row_start", c.row_start.clone()),
                        ("table", c.table.clone()), ("n_seqs", 2), ("width", 4), ("device", torch.device("cpu", 1))):
        with pytest.raises(AttributeError, match=name):
            setattr(c, name, value)
        with pytest.raises(AttributeError, match=name):
            delattr(c, name)
    after = struct(c, kv, 7)
    assert bytes(after) == bytes(before) and after.table == c.table.data_ptr()


def test_a_chunks_tensors_change_in_place():
    c, kv = chunk(), cache()
    c.ctx_len += 3                                     # in place: the same tensor, read when the kernels run
    c.table[0, 0] = 7
    assert c.ctx_len.tolist() == [3, 3, 3] and struct(c, kv, 1).ctx_len == c.ctx_len.data_ptr()


def test_a_chunk_keeps_few_structures():
    c = chunk()
    for page in (32, 64):
        kv = cache(page)
        for n in range(2000):
            s = struct(c, kv, n)
            assert s.n_rows == n and s.max_len == 5 * page
    assert sum(len(x) for x in vars(c).values() if isinstance(x, dict)) <= 64


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
def test_a_paged_cache_does_not_change_under_its_calls(dtype):
    kv = cache(dtype=dtype)
    before, held = bytes(kv.struct), [kv.k, kv.v, kv.k_scales, kv.v_scales]
    for name, value in (("k", kv.k.clone()), ("v", kv.v.clone()), ("k_scales", dev(torch.zeros(1))), ("v_scales", dev(torch.zeros(1))),
                        ("n_pages", 4), ("page_size", 32), ("n_kv_heads", 1), ("head_dim", 128), ("kvq", "none"),
                        ("device", torch.device("cpu", 1))):
        with pytest.raises(AttributeError, match=name):
            setattr(kv, name, value)
    assert bytes(kv.struct) == before and all(a is b for a, b in zip(held, [kv.k, kv.v, kv.k_scales, kv.v_scales]))
    kv.k += 1                                          # contents may change
    assert kv.struct.k == kv.k.data_ptr()


def test_a_chunks_default_bound_is_one_that_the_entries_take():
    kv = fp.PagedKV(dev(torch.zeros(1, 1, 65536, 64, dtype=torch.int8)), dev(torch.zeros(1, 1, 2048, 64, 32, dtype=torch.int8)),
                    *[dev(torch.zeros(1, 1, 65536, dtype=torch.float16)) for _ in range(2)])
    i = dev(torch.zeros(2, dtype=torch.int32))
    c = fp.Chunk(i, i[:1], dev(torch.zeros(1, 40000, dtype=torch.int32)), max_new=1)
    assert struct(c, kv, 1).max_len == 2**31 - 1024
