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
