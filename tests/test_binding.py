"""What the Python binding takes for pointers, rows and index arrays."""
import pytest
import torch

from paper_2307_15517_amd import mx


def test_anything_with_a_data_pointer_is_a_pointer():
    """Tensors, parameters, storages, integers and None, as far as the check of the sizes (no launch follows)."""
    x = torch.zeros(1024)
    for p in (x, torch.nn.Parameter(x), x.untyped_storage(), x.data_ptr(), None):
        for call in (lambda: mx.mx_dequantize(p, p, 1, -1, 32, mx.fmt(32, 8), p, stream=0),
                     lambda: mx.mx_cache_append(p, p, mx.MX_F32, -1, 64, 64, mx.cache_format(1, 16, 1, 64), p, p, p, p, p, stream=0)):
            with pytest.raises(mx.MxError) as e:
                call()
            assert e.value.status == mx.MX_ERR_BAD_ARG


@pytest.mark.gpu
def test_index_arrays_and_outputs_elsewhere_are_refused():
    """A slot array on the host or with gaps, an output on the host: refused before the call, and nothing is written."""
    dev = "cuda:0"
    cache = mx.Cache(4, 16, 2, 64, mx.fmt(32, 8), dev)
    x = torch.ones((8, 128), device=dev)
    slots = torch.arange(16, dtype=torch.int32, device=dev)
    for bad in (slots[:8].cpu(), slots[::2], slots[:8].long(), slots[:7]):
        with pytest.raises(AssertionError):
            mx.cache_append(cache, x, x, bad)
    assert not cache.k.any() and not cache.v.any()
    mx.cache_append(cache, x, x, slots[:8])
    table, q_start, kv_len = (torch.tensor(t, dtype=torch.int32, device=dev) for t in ([[0, 1]], [0, 8], [8]))
    for out in (torch.empty((8, 256)), torch.empty((8, 256), device=dev, dtype=torch.bfloat16), torch.empty((8, 512), device=dev)[:, ::2]):
        with pytest.raises(AssertionError):
            mx.cache_attention(cache, x.repeat(1, 2), table, q_start, kv_len, 8, 8, out=out)
    for bad in (table.cpu(), table.long(), table.repeat(1, 2)[:, ::2]):
        with pytest.raises(AssertionError):
            mx.cache_attention(cache, x.repeat(1, 2), bad, q_start, kv_len, 8, 8)
    assert bool((mx.cache_attention(cache, x.repeat(1, 2), table, q_start, kv_len, 8, 8) == 1.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_single_row_of_any_stride(dtype):
    """One new token whose row comes from a column: its stride from row to row is one element, and means nothing."""
    dev = "cuda:0"
    cache = mx.Cache(1, 16, 2, 64, None, dev)
    x = torch.randn((128, 1), device=dev).to(dtype).t()
    assert x.shape == (1, 128) and x.stride() == (1, 1)
    mx.cache_append(cache, x, x, torch.tensor([3], dtype=torch.int32, device=dev))
    assert torch.equal(cache.k.view(torch.bfloat16).reshape(2, 16, 64)[:, 3].reshape(1, 128), x.to(torch.bfloat16))
    table, q_start, kv_len = (torch.tensor(t, dtype=torch.int32, device=dev) for t in ([[0]], [0, 1], [4]))
    q = torch.randn((128, 1), device=dev).to(dtype).t()
    out = torch.empty((128, 1), device=dev, dtype=dtype).t()
    got = mx.cache_attention(cache, q, table, q_start, kv_len, 1, 4, out=out)
    assert got is out and torch.equal(out, mx.cache_attention(cache, q.clone(memory_format=torch.contiguous_format), table, q_start, kv_len, 1, 4))
