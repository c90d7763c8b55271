"""Calls on a stream that is not the current one, while the current one is at work: neither gets the other's memory."""
import types

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

SLEEP = 60_000_000      # cycles: some 30 ms


def _b():
    from paper_1905_05686_b200 import binding
    return binding


def tensors(out):
    """The tensors of a call's result."""
    if isinstance(out, torch.Tensor):
        return [out]
    if isinstance(out, (tuple, list)):
        return [t for o in out for t in tensors(o)]
    return [getattr(out, name) for name in type(out).__slots__ if isinstance(getattr(out, name), torch.Tensor)]


def calls(seed):
    """name -> call(stream) of each call that makes its outputs, on inputs of its own."""
    b = _b()
    g = torch.Generator("cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda").bfloat16()
    x, dy, gamma = normal(700, 1000), normal(700, 1000), torch.ones(1000, device="cuda")
    _, mean, rstd, kept = b.lrbi_layer_norm(x, gamma, checkpoint=True)
    W = normal(512, 640)
    w4, X = b.lrbi_w4_quantize((512, 640, 512, 640, 1), W), normal(6, 640)
    return {
        "store": lambda s: b.lrbi_checkpoint_store(x, stream=s),
        "load": lambda s: b.lrbi_checkpoint_load(kept, stream=s),
        "norm": lambda s: b.lrbi_layer_norm(x, gamma, checkpoint=True, stream=s),
        "norm_backward": lambda s: b.lrbi_layer_norm_backward(dy, kept, gamma, mean, rstd, restore=True, stream=s),
        "activation": lambda s: b.lrbi_activation(x, "gelu", checkpoint=True, stream=s),
        "activation_backward": lambda s: b.lrbi_activation_backward(dy, kept, "gelu", restore=True, stream=s),
        "quantize": lambda s: b.lrbi_w4_quantize((512, 640, 512, 640, 1), W, stream=s),
        "product": lambda s: b.lrbi_w4_gemv(w4, X, stream=s),
    }


NAMES = ["store", "load", "norm", "norm_backward", "activation", "activation_backward", "quantize", "product"]


def held(out):
    """Bytes of the allocations behind a result."""
    return list({t.untyped_storage().data_ptr(): t.untyped_storage().nbytes() for t in tensors(out)}.values())


@pytest.mark.parametrize("name", NAMES)
def test_memory_that_the_current_stream_still_reads(name):
    """Blocks of the sizes that the call needs are freed while the current stream has yet to read them."""
    call = calls(1)[name]
    want = call(None)
    sizes = held(want)
    side = torch.cuda.Stream()
    call(side)                      # that stream's pool has room now: memory asked of the driver later waits for the device
    blocks = [torch.full((n,), 37, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
    torch.cuda.synchronize()
    torch.cuda._sleep(SLEEP)
    copies = [t.clone() for t in blocks]
    places = {t.data_ptr() for t in blocks}
    del blocks
    got = call(side)
    assert not places & {t.untyped_storage().data_ptr() for t in tensors(got)}
    side.synchronize()
    assert not torch.cuda.current_stream().query()          # the current stream has not come to its copies yet
    torch.cuda.synchronize()
    assert all((c == 37).all() for c in copies)
    assert all(torch.equal(p, q) for p, q in zip(tensors(got), tensors(want)))


@pytest.mark.parametrize("name", NAMES)
def test_results_that_the_current_stream_still_reads(name):
    """Results are freed while the current stream has yet to read them, and the call is made again on the other stream."""
    call, other = calls(1)[name], calls(2)[name]
    want = tensors(call(None))
    side = torch.cuda.Stream()
    room = [call(side) for _ in range(6)]
    del room
    torch.cuda.synchronize()
    got = tensors(call(side))
    side.synchronize()
    torch.cuda._sleep(SLEEP)
    copies = [t.clone() for t in got]
    del got
    again = [other(side) for _ in range(3)]
    side.synchronize()
    assert not torch.cuda.current_stream().query()
    torch.cuda.synchronize()
    assert all(torch.equal(c, t) for c, t in zip(copies, want))
    assert all(torch.equal(p, q) for a in again for p, q in zip(tensors(a), tensors(other(None))))


def test_the_current_stream_given_by_name():
    b = _b()
    x = torch.randn((40, 264), device="cuda")
    a = b.lrbi_activation(x, "silu", stream=torch.cuda.current_stream())
    assert torch.equal(a, b.lrbi_activation(x, "silu"))


def test_streams_of_another_device_are_refused():
    b = _b()
    x = torch.zeros((4, 40), device="cuda")
    for device, kind in ((1, 1), (0, 0)):
        with pytest.raises(ValueError):
            b.lrbi_activation(x, "relu", stream=types.SimpleNamespace(stream_id=0, device_index=device, device_type=kind))
