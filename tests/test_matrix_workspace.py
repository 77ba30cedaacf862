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


@pytest.mark.parametrize("n, k", [(-1, 3), (2, -3), (-2, -3), (0, 3), (2, 0)])
def test_counts_of_messages_that_are_none_are_refused(n, k):
    """A negative count is a large one to the library, and no tensor is too short for its product."""
    import paper_2005_10761_amd as rt
    t = torch.zeros(4, 6)
    with pytest.raises(ValueError, match="at least 1"):
        rt.aggregate_update_orthogonal([t], [t], n, k, 0.1, 1.0, 0.9, [t], [t])
