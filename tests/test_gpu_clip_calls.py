"""The life of a list of gradients: destroyed lists, streams, memory."""
import pytest
import torch

from paper_2012_05396_b200 import binding as B
from paper_2012_05396_b200 import layers as L

pytestmark = pytest.mark.gpu


def test_a_destroyed_list_is_refused():
    a = torch.full((64,), 2.0, device="cuda")
    lst = L.GradList([a])
    assert float(L.ssd_clip_grad_norm(lst, 8.0)) == 16.0
    clipped = a.clone()
    assert bool((clipped < 2.0).all())
    lst.ssd_grad_list_destroy()
    for call in (lambda: L.ssd_clip_grad_norm(lst, 1.0), lambda: L.ssd_grad_norm(lst)):
        with pytest.raises(B.SsdError) as e:
            call()
        assert e.value.status == B.SSD_ERR_ARG
    lst.ssd_grad_list_destroy()
    assert torch.equal(a, clipped)


def allocated_on(tensor):
    """The stream whose memory a tensor lies in, by the allocator's own account."""
    at = tensor.data_ptr()
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= at < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not in any segment")


@pytest.mark.parametrize("raw", [False, True])
def test_the_table_is_memory_of_the_stream_that_fills_it(raw):
    """Blocks that work pending on one stream still uses are free for that stream alone: a table filled on another must not be cut from them."""
    g = [torch.full((5000,), 3.0, device="cuda"), torch.full((700,), 4.0, device="cuda")]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lst = L.GradList(g, groups=[0, 1], stream=side.cuda_stream if raw else side)
    assert allocated_on(lst._keep[2]) == side.cuda_stream
    assert allocated_on(L.GradList(g)._keep[2]) == torch.cuda.current_stream().cuda_stream
    # the table is in place when the list is: a call on any stream may follow
    norms = L.ssd_grad_norm(lst)
    assert torch.allclose(norms, torch.tensor([3.0 * 5000 ** 0.5, 4.0 * 700 ** 0.5], device="cuda"), rtol=1e-6)
