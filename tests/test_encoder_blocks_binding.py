"""What the binding refuses of an encoder's gated blocks before it calls the library: blocks of another width, on another device, gradients that would be written past their ends."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2506_01084_amd import api  # noqa: E402


class Nothing:
    """A library that is not to be called."""

    def __getattr__(self, name):
        def call(*args):
            raise RuntimeError(f"{name} was called")
        return call


def _context(d=128):
    ctx = object.__new__(api.Context)
    ctx._lib, ctx._h, ctx._device = Nothing(), None, 0
    ctx.B, ctx.V, ctx.M, ctx.cap, ctx.d, ctx.dtype, ctx.torch_dtype = 2, 50, 3, 20, d, "bf16", torch.bfloat16
    return ctx


def _block(d=128, d_ff=64, group=0, device="cuda:0"):
    block = object.__new__(api.GatedFFN)
    block.tensors, block.device, block.d, block.d_ff = (), torch.device(device), d, d_ff
    block.desc = api.FfnDesc()
    block.desc.d_ff, block.desc.group = d_ff, group
    return block


def _encoder(*blocks):
    return api.Encoder(dict(n_heads=2, attention_only=False, pos=None, layers=[{} for _ in blocks], ffn=list(blocks)), torch.bfloat16)


E, W, dE = torch.zeros((50, 128), dtype=torch.bfloat16), torch.zeros((2, 20, 128), dtype=torch.bfloat16), torch.zeros((50, 128))

BAD = [(AssertionError, dict(d=64)), (AssertionError, dict(d=192)), (ValueError, dict(device="cuda:1"))]


@pytest.mark.parametrize("error,kw", BAD)
@pytest.mark.parametrize("where", [0, 1])
def test_blocks_of_another_width_or_device(error, kw, where):
    ctx = _context()
    blocks = [_block(), _block()]
    blocks[where] = _block(**kw)
    bad, good = _encoder(*blocks), _encoder(_block(), _block())
    match = "expected weights on cuda:0" if error is ValueError else None
    with pytest.raises(error, match=match):
        ctx.hyper_encode(E, bad, W)
    with pytest.raises(error, match=match):
        ctx.hyper_encode_keep(E, bad, W)
    with pytest.raises(error, match=match):
        ctx.hyper_encode_backward(E, bad, W, good, dE)
    with pytest.raises(error, match=match):
        ctx.hyper_encode_backward(E, good, W, bad, dE)


@pytest.mark.parametrize("grad", [[dict(d_ff=128), {}], [{}, dict(group=32)], [{}, dict(d_ff=32)], [{}], [{}, {}, {}]])
def test_gradients_of_other_shapes(grad):
    with pytest.raises(AssertionError):
        _context().hyper_encode_backward(E, _encoder(_block(), _block()), W, _encoder(*[_block(**kw) for kw in grad]), dE)


def test_others_go_on_to_the_tensors():
    """(These checks pass; what is refused next is that the tensors are not on a device.)"""
    ctx, good = _context(), _encoder(_block(), _block())
    for call in (lambda: ctx.hyper_encode(E, good, W), lambda: ctx.hyper_encode_keep(E, good, W), lambda: ctx.hyper_encode_backward(E, good, W, _encoder(_block(), _block()), dE),
                 lambda: ctx.hyper_encode(E, _encoder(_block(group=32)), W)):
        with pytest.raises(ValueError, match="contiguous device tensor"):
            call()
    assert ctypes.addressof(good.desc) == ctypes.addressof(good._gated)
