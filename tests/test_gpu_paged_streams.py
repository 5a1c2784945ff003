"""Rotary and paged objects whose HIP stream is not the current one at the call: who owns new outputs, and how long memory that the call was
given is kept."""
import pytest
import torch

from paper_2409_09086_amd import binding as B
from test_gpu_paged import DEV, Case

pytestmark = pytest.mark.gpu


def owner(t):
    """The HIP stream that a tensor's memory goes back to."""
    at = t.data_ptr()
    return next(x["stream"] for x in torch.cuda.memory_snapshot() if x["address"] <= at < x["address"] + x["total_size"])


def made(side):
    c = Case(31, "bf16", 8, 2, 128, 16, [(64, 300), (1, 200)])
    with torch.cuda.stream(side):
        cache, rot = c.cache(), B.Rotary(128, 512)
    K, V, b = c.K.to(DEV), c.V.to(DEV), c.batch()
    side.wait_stream(torch.cuda.current_stream())
    return c, cache, rot, K, V, b


def calls(c, cache, rot, K, V, b, q, k, v):
    """The calls that make and read tensors, by name."""
    pos = torch.arange(c.tokens, dtype=torch.int32, device=DEV)
    return {"apply": lambda: rot.apply(pos, q, k)[0], "append": lambda: cache.append(b, k, v, K, V, rotary=rot, q=q),
            "attend": lambda: cache.attend(b, q, K, V)}


@pytest.mark.parametrize("name", ["apply", "append", "attend"])
def test_new_outputs_belong_to_the_objects_stream(name):
    """A dropped output's memory goes back to the stream that writes it, not to the current one, which may hand it on at once."""
    side = torch.cuda.Stream()
    args = made(side)
    c = args[0]
    q, k, v = (x.to(DEV).contiguous() for x in (c.q, c.k, c.v))
    want = calls(*args, q, k, v)[name]()                       # warm: the allocator has blocks of every size on both streams
    side.synchronize()
    want = want.clone()
    torch.cuda.synchronize()
    side.wait_stream(torch.cuda.current_stream())
    out = calls(*args, q, k, v)[name]()
    assert owner(out) == side.cuda_stream != owner(q)
    side.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("name", ["apply", "append", "attend"])
def test_dropped_inputs_live_until_the_call_has_run(name):
    """While the object's stream is busy elsewhere, the memory of dropped inputs is not handed on."""
    side = torch.cuda.Stream()
    args = made(side)
    c = args[0]
    q, k, v = (x.to(DEV).contiguous() for x in (c.q, c.k, c.v))
    K0, V0 = args[3].clone(), args[4].clone()
    torch.cuda.synchronize()
    want = calls(*args, q, k, v)[name]()
    side.synchronize()
    args[3].copy_(K0), args[4].copy_(V0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)                         # some 170 ms, the calls below take less than one
    out = calls(*args, q, k, v)[name]()
    held = {q.data_ptr(), k.data_ptr()} | ({v.data_ptr()} if name == "append" else set())
    held -= {k.data_ptr()} if name == "attend" else set()
    del q, k, v
    new = [torch.empty((c.tokens, h, 128), dtype=torch.bfloat16, device=DEV) for h in (8, 8, 2, 2, 2, 2)]
    taken = held & {x.data_ptr() for x in new}
    busy = not side.query()                                    # and was so all the while
    for x in new:
        x.fill_(float("nan"))
    side.synchronize()
    assert not (busy and taken)
    assert torch.equal(out, want)


def test_the_workspace_belongs_to_the_objects_stream():
    side = torch.cuda.Stream()
    c = Case(32, "bf16", 8, 2, 128, 16, [(1, 40)])
    cache = c.cache(hip_stream=side.cuda_stream)
    assert owner(cache.workspace) == side.cuda_stream
    side.synchronize()


def test_under_the_objects_own_stream_nothing_is_kept():
    """The usual call: outputs and inputs are recycled in stream order, as ever."""
    side = torch.cuda.Stream()
    args = made(side)
    c = args[0]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()                                   # nothing waits for an event of an earlier test
    waiting = lambda: torch.cuda.memory_stats()["active_bytes.all.current"] - torch.cuda.memory_stats()["allocated_bytes.all.current"]
    before = waiting()
    with torch.cuda.stream(side):
        q, k, v = (x.to(DEV).contiguous() for x in (c.q, c.k, c.v))
        for name in ("apply", "append", "attend"):
            calls(*args, q, k, v)[name]()
        del q, k, v
        assert waiting() == before
    side.synchronize()
