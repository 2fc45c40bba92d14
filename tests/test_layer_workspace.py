"""The workspace that a call of layers.py makes belongs to the stream that uses it."""
import contextlib

import pytest
import torch

from paper_2605_08565_amd import layers


class Stream:
    """What the Python form asks of a stream."""
    cuda_stream = 7


def test_it_is_allocated_on_the_stream_of_the_call(monkeypatch):
    """No GPU needed: the current stream at the moment of the allocation is the call's, and what was current before is after."""
    current = ["current"]
    made = []

    @contextlib.contextmanager
    def stream(s):
        current.append(s)
        yield
        current.pop()

    class Tensor:
        def record_stream(self, s):
            pass

    def empty(*args, **kw):
        made.append(current[-1])
        return Tensor()
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch, "empty", empty)
    side = Stream()
    layers._workspace(64, "cpu", None)
    layers._workspace(64, "cpu", side)
    assert made == ["current", side] and current == ["current"]


@pytest.mark.gpu
def test_memory_freed_on_a_busy_stream_is_not_the_workspace_of_another():
    """The current stream is held and then writes blocks of the workspace's size, which the host has freed meanwhile; a call on an idle
    stream has the result that it always has."""
    from paper_2605_08565_amd import mxq
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    m, k, n = 24, 4096, 2048
    x = torch.randn((m, k), generator=gen, device="cuda").bfloat16()
    codes, scales, _ = mxq.quantize(torch.randn((n, k), generator=gen, device="cuda").bfloat16(), 32, mxq.SCALE_E8M0, mxq.RECIPE_ABSMAX)
    w = layers.W4(codes, scales, 32, mxq.SCALE_E8M0)
    ad = layers.Adapters(torch.randn((5, 16, k), generator=gen, device="cuda").bfloat16(),
                         torch.randn((5, n, 16), generator=gen, device="cuda").bfloat16(), torch.ones(5, device="cuda"))
    ids = (torch.arange(m, device="cuda") % 5).int()
    want = layers.linear(x, w, ad, ids)
    out = torch.empty_like(want)
    # Streams share a few hardware queues: one that shares the held stream's waits for it, and shows nothing; of four, some do not.
    for side in [torch.cuda.Stream() for _ in range(4)]:
        torch.cuda.synchronize()
        layers.linear(x, w, ad, ids, out=out, stream=side)            # what the side stream needs of its own is there
        side.synchronize()
        out.zero_()
        blocks = [torch.empty(1 << s, device="cuda", dtype=torch.uint8) for s in range(9, 25) for _ in range(3)]
        torch.cuda.synchronize()
        torch.cuda._sleep(100_000_000)
        for b in blocks:
            b.fill_(255)                                              # NaN wherever a float is read from it
        del blocks, b
        layers.linear(x, w, ad, ids, out=out, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
