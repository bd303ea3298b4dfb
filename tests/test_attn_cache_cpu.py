"""What a KVCache hands to a call is what it holds at that call."""
import ctypes

import pytest
import torch

from paper_2506_04985_b200 import binding as B


@pytest.fixture(autouse=True, scope="module")
def built():
    from paper_2506_04985_b200 import build
    build.build()


def struct(c):
    return B._KVCacheStruct.from_buffer_copy(c.ref)


def a_cache(n_pages=3, seqs=2, width=2):
    k = torch.zeros((n_pages, 2, 16, 64), dtype=torch.int8)
    s = torch.zeros((n_pages, 2))
    return B.KVCache(k, k.clone(), s, s.clone(), torch.zeros((seqs, width), dtype=torch.int32))


def test_another_page_table_takes_effect():
    c = a_cache()
    bigger = torch.zeros((5, 9), dtype=torch.int32)
    c.pages = bigger
    assert c.n_seqs == 5 and struct(c).pages == bigger.data_ptr() and struct(c).max_pages == 9
    assert (c.n_kv, c.head_dim, c.dev) == (2, 64, -1)


def test_other_storage_takes_effect():
    c, other = a_cache(), a_cache(n_pages=10)
    c.k, c.v, c.k_scale, c.v_scale = other.k, other.v, other.k_scale, other.v_scale
    s = struct(c)
    assert s.n_pages == 10
    assert [s.k, s.v, s.k_scale, s.v_scale] == [t.data_ptr() for t in (other.k, other.v, other.k_scale, other.v_scale)]


def test_a_tensor_given_other_memory_takes_effect():
    c = a_cache()
    c.pages.resize_(64, 64)
    assert struct(c).pages == c.pages.data_ptr() and struct(c).max_pages == 64 and c.n_seqs == 64


def test_what_is_no_cache_any_more_is_refused():
    c = a_cache()
    c.pages = c.pages.long()
    assert c.ref is None
    c = a_cache()
    c.k = None
    assert c.ref is None
    with pytest.raises(TypeError):
        B.KVCache.heads("two", 64)
    bare = B.KVCache.heads(2, 64)
    assert (bare.n_seqs, bare.n_kv, bare.head_dim, bare.dev) == (0, 2, 64, -1) and not struct(bare).k
    assert ctypes.sizeof(B._KVCacheStruct) == len(bare.ref)
