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


def test_views_that_do_not_fit_leave_nothing(reader):
    """A buffer too small for the last of the results: an error, and the views that were made are given back."""
    def tensors():
        gc.collect()
        return sum(type(o) is torch.Tensor for o in gc.get_objects())

    flat = torch.zeros(3 * 4 + 4 + 4 + 2 * 4)  # (without room for the ids)
    reader.views(torch.zeros(100), 4, True, True, 2)
    was = tensors()
    for _ in range(20):
        with pytest.raises(RuntimeError):
            reader.views(flat, 4, True, True, 2)
    assert tensors() == was
    with pytest.raises(TypeError):
        reader.views(None, 4, True, True, 2)


@pytest.mark.parametrize("given,entropy,top", [(False, False, 0), (True, False, 3), (False, True, 1), (True, True, 2)])
def test_views(reader, given, entropy, top):
    n = 4
    flat = torch.arange(n * (3 + given + entropy + 2 * top), dtype=torch.float32)
    stats, lse, log_prob, h, top_log_probs, top_ids = reader.views(flat, n, given, entropy, top)
    want = list(flat.split([2 * n, n, n * given, n * entropy, n * top, n * top]))
    assert torch.equal(stats, want[0].view(n, 2)) and torch.equal(lse, want[1])
    assert torch.equal(log_prob, want[2]) if given else log_prob is None
    assert torch.equal(h, want[3]) if entropy else h is None
    if top:
        assert torch.equal(top_log_probs, want[4].view(n, top))
        assert torch.equal(top_ids, want[5].view(torch.int32).view(n, top))
    else:
        assert top_log_probs is None and top_ids is None
