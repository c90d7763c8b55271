"""Calls on a stream that is not the current one, while the current one is at work: neither gets the other's memory."""
import types

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_1905_05686_b200 import synth

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
    layer = synth.Layer("streams", 512, 640, 128, 128, 16, 0.3, 0.05)
    Ip, Iz = synth.make_factors(layer)
    ip, iz = b.to_device_words(synth.pack_ip(Ip)), b.to_device_words(synth.pack_iz(Iz))
    Wt, many, dY = b.lrbi_transpose_bf16(W), normal(200, 640), normal(200, 512)
    mp, mz = torch.rand((20, 128, 16), generator=g, device="cuda"), torch.rand((20, 16, 128), generator=g, device="cuda")
    half = torch.full((20,), 0.5, device="cuda")
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
        "mask": lambda s: b.lrbi_decode_mask(layer, ip, iz, stream=s),
        "masks": lambda s: b.lrbi_decode_mask_batch([layer, layer], [ip, ip], [iz, iz], stream=s),
        "masked": lambda s: b.lrbi_masked_gemm(layer, W, ip, iz, many, stream=s),
        "transpose": lambda s: b.lrbi_transpose_bf16(W, stream=s),
        "dx": lambda s: b.lrbi_masked_gemm_dx(layer, Wt, ip, iz, dY, stream=s),
        "dw": lambda s: b.lrbi_masked_gemm_dw(layer, dY, many, ip, iz, stream=s),
        "threshold": lambda s: b.lrbi_threshold_pack(layer, mp, mz, half, half, stream=s),
        "cost": lambda s: b.lrbi_index_cost(layer, W, 0.05, ip, iz, stream=s),
    }


NAMES = ["store", "load", "norm", "norm_backward", "activation", "activation_backward", "quantize", "product", "mask", "masks", "masked", "transpose",
         "dx", "dw", "threshold", "cost"]


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


@pytest.mark.parametrize("name", ["dw", "nmf"])
def test_workspaces(name):
    """The same for the scratch of the two calls whose workspace the binding makes."""
    import ctypes
    b = _b()
    layer = synth.Layer("streams", 512, 640, 128, 128, 16, 0.3, 0.05)
    lay = b.Layout.of(layer)
    mp, mz = torch.rand((20, 128, 16), device="cuda"), torch.rand((20, 16, 128), device="cuda")
    W = torch.randn((512, 640), device="cuda").bfloat16()
    factors = [(mp.clone(), mz.clone()) for _ in range(3)]
    if name == "dw":
        need, call = b.lib().lrbi_masked_gemm_dw_workspace(ctypes.byref(lay), 200), lambda i, s: calls(1)["dw"](s)
    else:
        need, call = b.lib().lrbi_nmf_workspace(ctypes.byref(lay)), lambda i, s: b.lrbi_nmf_update(layer, W, *factors[i], 3, stream=s)
    side = torch.cuda.Stream()
    want = tensors(call(0, None))
    call(1, side)
    blocks = [torch.full((need,), 37, dtype=torch.uint8, device="cuda") for _ in range(2)]
    made = calls(1)["dw"] if name == "dw" else None
    torch.cuda.synchronize()
    torch.cuda._sleep(SLEEP)
    copies = [t.clone() for t in blocks]
    del blocks
    got = tensors(made(side) if made else call(2, side))
    side.synchronize()
    assert not torch.cuda.current_stream().query()
    torch.cuda.synchronize()
    assert all((c == 37).all() for c in copies) and all(torch.equal(p, q) for p, q in zip(got, want))


def test_the_current_stream_given_by_name():
    b = _b()
    x = torch.randn((40, 264), device="cuda")
    a = b.lrbi_activation(x, "silu", stream=torch.cuda.current_stream())
    assert torch.equal(a, b.lrbi_activation(x, "silu"))


def test_streams_that_torch_did_not_make():
    """Calls that take a stream by its handle go on taking any object that has one."""
    b = _b()
    W = torch.randn((64, 96), device="cuda").bfloat16()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for handle in (side.cuda_stream, torch.cuda.current_stream().cuda_stream):
        got = b.lrbi_transpose_bf16(W, stream=types.SimpleNamespace(cuda_stream=handle))
        torch.cuda.synchronize()
        assert torch.equal(got, W.t())


def test_streams_of_another_device_are_refused():
    b = _b()
    x = torch.zeros((4, 40), device="cuda")
    for device, kind in ((1, 1), (0, 0)):
        with pytest.raises(ValueError):
            b.lrbi_activation(x, "relu", stream=types.SimpleNamespace(stream_id=0, device_index=device, device_type=kind))
