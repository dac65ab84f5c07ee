"""A step's arrays: taken as they are where calls are to follow them, copied where the step is made from host lengths."""
import pytest
import torch

from paper_2609_34060_amd import kvc

DEV = "cuda"


def i32(*x, device="cpu"):
    return torch.tensor(x, dtype=torch.int32, device=device)


def test_tables_on_the_device_are_taken_as_they_are():
    """A copy would not be followed by a captured call: tables of another type or layout are refused."""
    wide = torch.arange(12, dtype=torch.int32).view(2, 6)
    step = kvc.Step.on_device(i32(0, 1, 2), i32(3, 4), 2, 1, 4, wide)
    assert step.tables is wide and step.c.tables == wide.data_ptr() and step.c.max_blocks == 6
    for bad in (wide.long(), wide.float(), wide[:, :3], wide[:, ::2], wide.t()[:2], wide[:1], wide[0]):
        with pytest.raises(ValueError, match="tables"):
            kvc.Step.on_device(i32(0, 1, 2), i32(3, 4), 2, 1, 4, bad)
    for other in (wide.long(), wide[:, :3], wide[:, ::2]):
        step = kvc.Step([1, 1], [3, 4], other)
        assert step.tables.is_contiguous() and step.tables.dtype == torch.int32 and torch.equal(step.tables.long(),
                                                                                                other.long())


@pytest.mark.gpu
def test_captured_calls_follow_tables():
    """Blocks that a table gets after the capture are those that replays read."""
    d, n = 64, 3
    g = torch.Generator().manual_seed(1)
    k, v = torch.randn(2, 12, 16, 2, d, generator=g).to(torch.bfloat16).to(DEV)
    cache = kvc.Cache([k], [v])
    tables = torch.arange(12, dtype=torch.int32, device=DEV).view(n, 4)
    starts, ctx = i32(0, 1, 2, 3, device=DEV), i32(20, 64, 33, device=DEV)
    step = kvc.Step.on_device(starts, ctx, n, 1, 64, tables)
    q = torch.randn(n, 4, d, generator=g).to(torch.bfloat16).to(DEV)
    out = torch.empty_like(q)
    ws = torch.empty(max(1, kvc.kvc_attend_workspace_bytes(cache, step, 4)), dtype=torch.uint8, device=DEV)
    kvc.kvc_attend(cache, step, q, out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvc.kvc_attend(cache, step, q, out, workspace=ws)
    for seed in range(4):
        order = torch.randperm(12, generator=g).to(torch.int32).view(n, 4)
        tables.copy_(order)
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, kvc.kvc_attend(cache, kvc.Step([1] * n, [20, 64, 33], order.to(DEV)), q))


@pytest.mark.gpu
def test_copied_tables_are_whole_on_every_stream():
    """A step made behind work of the current stream, from tables that are converted, and used on another stream at once."""
    d, width = 64, 1 << 24
    g = torch.Generator().manual_seed(2)
    k, v = torch.randn(2, 8, 16, 2, d, generator=g).to(torch.bfloat16).to(DEV)
    cache = kvc.Cache([k], [v])
    q = torch.randn(1, 4, d, generator=g).to(torch.bfloat16).to(DEV)
    want = kvc.kvc_attend(cache, kvc.Step([1], [100]), q)
    tables = torch.full((1, width), -1, dtype=torch.int64, device=DEV)
    at = width - 8  # the sequence's blocks are the last ones of its row
    tables[0, at:] = torch.arange(8, device=DEV)
    side = torch.cuda.Stream()
    gone = torch.full((1, width), -1, dtype=torch.int32, device=DEV)  # (what the converted tables' memory held before)
    torch.cuda.synchronize()
    del gone
    torch.cuda._sleep(20_000_000)
    step = kvc.Step([1], [100], tables, offsets=[at * 16])
    out = kvc.kvc_attend(cache, step, q, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.gpu
@pytest.mark.parametrize("host", ["k_pools", "v_pools", "k_scales", "v_scales"])
def test_caches_with_a_part_in_host_memory(host):
    """Refused by all three calls: the kernels would be given an address that is none of theirs."""
    parts = {n: [torch.zeros(4, 16, 2, 64, dtype=torch.int8, device=DEV) if "pools" in n else
                 torch.zeros(4, 16, 2, device=DEV) for _ in range(2)] for n in ("k_pools", "v_pools", "k_scales", "v_scales")}
    good = kvc.Cache(**parts)
    parts[host][1] = parts[host][1].cpu()
    bad = kvc.Cache(**parts)
    step = kvc.Step([3], [5], device=DEV)
    k = torch.randn(2, 3, 2, 64, device=DEV).to(torch.bfloat16)
    for call in (kvc.kvc_append, kvc.kvc_gather):
        call(good, step, k, k.clone())
        with pytest.raises(ValueError, match="one GPU"):
            call(bad, step, k, k.clone())
    q = torch.randn(3, 4, 64, device=DEV).to(torch.bfloat16)
    kvc.kvc_attend(good, step, q)
    with pytest.raises(ValueError, match="one GPU"):
        kvc.kvc_attend(bad, step, q)
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_calls_run_on_the_current_gpu(monkeypatch):
    """Another current device, or a stream of another, is refused: the kernels would run there."""
    pool = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16, device=DEV)
    cache, step = kvc.Cache([pool], [pool.clone()]), kvc.Step([3], [5], device=DEV)
    k = torch.randn(3, 2, 64, device=DEV).to(torch.bfloat16)
    q = torch.randn(3, 4, 64, device=DEV).to(torch.bfloat16)

    class Elsewhere:
        device_index, cuda_stream = 1, 0

    calls = [lambda **kw: kvc.kvc_append(cache, step, k, k.clone(), **kw),
             lambda **kw: kvc.kvc_gather(cache, step, k, k.clone(), **kw), lambda **kw: kvc.kvc_attend(cache, step, q, **kw)]
    for call in calls:
        call()
        call(stream=torch.cuda.Stream())
        with pytest.raises(ValueError, match="stream"):
            call(stream=Elsewhere())
        with monkeypatch.context() as m:
            m.setattr(torch._C, "_cuda_getDevice", lambda: 1)
            m.setattr(kvc, "_several_gpus", lambda: True)
            with pytest.raises(ValueError, match="current"):
                call()
    torch.cuda.synchronize()
