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
