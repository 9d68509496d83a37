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
    assert allocated_on(lst.table) == side.cuda_stream
    assert allocated_on(L.GradList(g).table) == torch.cuda.current_stream().cuda_stream
    # the table is in place when the list is: a call on any stream may follow
    norms = L.ssd_grad_norm(lst)
    assert torch.allclose(norms, torch.tensor([3.0 * 5000 ** 0.5, 4.0 * 700 ** 0.5], device="cuda"), rtol=1e-6)


def test_a_list_dropped_while_another_stream_uses_it():
    """The table's memory is not handed out again before the calls on it are done, whichever stream they run on."""
    n = 300000
    g = torch.full((n,), 2.0, device="cuda")
    norms = torch.empty(1, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    lst = L.GradList([g])
    at, size = lst.table.data_ptr(), lst.table.numel()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)              # a tenth of a second
    L.ssd_clip_grad_norm(lst, 1.0, norms=norms, stream=side)
    del lst
    assert not side.query()
    fresh = [torch.full((size,), 255, device="cuda", dtype=torch.uint8) for _ in range(8)]
    assert all(not (t.data_ptr() <= at < t.data_ptr() + size) for t in fresh)
    side.synchronize()
    assert abs(float(norms) - 2.0 * n ** 0.5) <= 1e-3
    assert torch.allclose(g, torch.full_like(g, n ** -0.5), rtol=1e-5)


def test_captured_into_a_graph():
    """A call captured on another stream than the list's, replayed on new gradients, and the list dropped afterwards."""
    g = torch.empty(40000, device="cuda")
    out = torch.empty(40000, device="cuda", dtype=torch.bfloat16)
    norms = torch.empty(2, device="cuda")
    lst = L.GradList([g[:30000], g[30000:]], out=[out[:30000], out[30000:]], groups=[0, 1])
    g.fill_(1.0)
    L.ssd_clip_grad_norm(lst, 2.0, norms=norms)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.ssd_clip_grad_norm(lst, 2.0, norms=norms)
    for v in (0.5, 8.0, 1e-3):
        g.fill_(v)
        graph.replay()
        want = torch.tensor([v * 30000 ** 0.5, v * 10000 ** 0.5], device="cuda")
        assert torch.allclose(norms, want, rtol=1e-6)
        for part, n in ((out[:30000], want[0]), (out[30000:], want[1])):
            f = min(1.0, 2.0 / (float(n) + 1e-6))
            assert torch.allclose(part.float(), torch.full_like(part, v * f, dtype=torch.float32), rtol=2.0 ** -8, atol=0)
    torch.cuda.synchronize()
    del graph, lst
    assert float(L.ssd_grad_norm(L.GradList([g]))) > 0


@pytest.mark.parametrize("sizes", [[5000] * 40, [3_000_000, 17, 40_000]], ids=["small", "large"])
@pytest.mark.parametrize("in_place", [False, True])
def test_gradients_written_by_the_kernel_before(sizes, in_place):
    """Every call sees what the kernel directly before it wrote, none of the values of the call before."""
    total = sum(sizes)
    arena, other = torch.empty(total, device="cuda"), torch.empty(total, device="cuda")
    views, at = [], 0
    for n in sizes:
        views.append((arena[at:at + n], other[at:at + n]))
        at += n
    lst = L.GradList([a for a, _ in views], out=None if in_place else [b for _, b in views])
    base = torch.randn(total, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    unit = base / float(base.double().norm())
    out = arena if in_place else other
    seen = []
    for i in range(200):
        torch.mul(base, float(1 + i % 7), out=arena)
        norm = L.ssd_clip_grad_norm(lst, 1.0)
        seen.append((norm, (out - unit).abs().max()))
    norms = torch.stack([n[0] for n, _ in seen]).double()
    want = float(base.double().norm()) * torch.tensor([1.0 + i % 7 for i in range(200)], dtype=torch.float64, device="cuda")
    # the products base * i and the factor round to float32 (2^-24 each); 1e-6 is added to norms of 400 and more
    assert bool(((norms - want).abs() <= 2.0 ** -21 * want).all())
    assert float(torch.stack([d for _, d in seen]).max()) <= 2.0 ** -20 * float(unit.abs().max())


def test_norms_over_what_a_call_uses_are_refused():
    arena, push = torch.full((4096,), 2.0, device="cuda"), torch.zeros(4096, device="cuda")
    lst = L.GradList([arena[1024:2048], arena[3000:3928]], out=[push[:1024], push[2048:2976]], groups=[0, 1])
    bad = [arena[1024:1026], arena[2046:2048], arena[2047:2049], arena[1023:1025], arena[3500:3502], push[0:2], push[1023:1025], push[2975:2977],
           lst.table[:8].view(torch.float32), lst.table[lst.table.numel() - 8:].view(torch.float32)]
    for norms in bad:
        for call in (lambda: L.ssd_clip_grad_norm(lst, 1.0, norms=norms), lambda: L.ssd_grad_norm(lst, norms=norms)):
            with pytest.raises(B.SsdError) as e:
                call()
            assert e.value.status == B.SSD_ERR_ARG
    assert bool((arena == 2.0).all()) and bool((push == 0.0).all())
    want = [2.0 * 1024 ** 0.5, 2.0 * 928 ** 0.5]
    for norms in (arena[1022:1024], arena[2048:2050], arena[2998:3000], arena[:2], arena[3928:3930], push[1024:1026], push[2046:2048], push[2976:2978]):
        assert L.ssd_clip_grad_norm(lst, 1.0, norms=norms) is not None
        assert torch.allclose(norms, torch.tensor(want, device="cuda"), rtol=1e-6)


def test_a_list_made_while_its_stream_is_captured():
    """Its table is filled when the graph runs, before the calls that the graph holds, with other kernels between them."""
    g, norms = torch.empty(70000, device="cuda"), torch.zeros(2, device="cuda")
    g.fill_(1.0)
    L.ssd_clip_grad_norm(L.GradList([g[:50000], g[50000:]], groups=[0, 1]), 1e9, norms=norms)      # the kernels are known to the device
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lst = L.GradList([g[:50000], g[50000:]], groups=[0, 1])
        g.mul_(2.0)
        L.ssd_clip_grad_norm(lst, 100.0, norms=norms)
    for v in (0.25, 1.0, 3.0):
        g.fill_(v)
        graph.replay()
        want = [2 * v * 50000 ** 0.5, 2 * v * 20000 ** 0.5]
        assert torch.allclose(norms, torch.tensor(want, device="cuda"), rtol=1e-6)
        for part, n in ((g[:50000], want[0]), (g[50000:], want[1])):
            assert torch.allclose(part, torch.full_like(part, 2 * v * min(1.0, 100.0 / (n + 1e-6))), rtol=1e-6)
    torch.cuda.synchronize()
    del graph, lst
