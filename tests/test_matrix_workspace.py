"""A workspace that the kernels cannot write to is refused by the binding of the matrix calls."""
import pytest
import torch

from paper_2005_10761_amd import binding


def test_a_workspace_in_host_memory_is_refused():
    """Its size and alignment may be right: the library has only the address, and its kernels would write there."""
    store = torch.empty(1 << 12, dtype=torch.uint8)
    at = -store.data_ptr() % 256
    with pytest.raises(TypeError):
        binding._workspace(store[at:at + 1024], 512, "cuda:0", None)


def test_no_workspace_is_taken_where_none_is_needed():
    assert binding._workspace(None, 0, "cuda:0", None) == (None, 0, None)
