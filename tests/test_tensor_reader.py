"""The binding's reader of tensors, on the CPU."""
import gc

import pytest
import torch


@pytest.fixture(scope="module")
def reader():
    import paper_2603_08957_amd as tre

    return tre.tre._reader()


def test_written_tensors_count_a_version(reader):
    """As torch's own in-place operations do; a tensor of inference mode has no count, and is left."""
    x, y = torch.zeros(3), torch.zeros(2, requires_grad=True)
    with torch.inference_mode():
        z = torch.zeros(2)
    reader.written([x, y, z])
    reader.written(y)
    reader.written((None,), None, x)
    assert (x._version, y._version) == (2, 2)
    with torch.inference_mode():
        reader.written([x, z])
    assert x._version == 3
    w = torch.ones(3, requires_grad=True)
    out = (w * w).sum()
    reader.written([w])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.backward()
    for bad in ([1], 5, "x"):
        with pytest.raises(TypeError):
            reader.written(bad)
