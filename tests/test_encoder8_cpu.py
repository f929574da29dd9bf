"""What an encoder in 8 bits takes from the encoder that it comes from, without a GPU: a context's stand-in lays weights out in plain torch."""
import pytest
import torch

from paper_2210_02574_amd.embedding import SentenceEncoder


class Weights:
    """Rows in 8 bits as HE.quantize8 makes them, on the CPU."""

    def quantize8(self, x, gelu=False):
        top = x.float().abs().amax(1)
        return torch.round(127 * x.float() / top[:, None]).to(torch.int8), top / 127


def _encoder(norm, dtype=torch.float32, slopes=None):
    layers = [SentenceEncoder.random_layer(16, 2, 24, 3 + i, dtype, "cpu") for i in range(2)]
    return SentenceEncoder(Weights(), layers, 2, norm=norm, last=torch.ones(16, dtype=dtype) if norm == "rms" else None, slopes=slopes)


def _tensors(encoder):
    out = [t for w in encoder.layers for v in w.values() for t in (v if isinstance(v, tuple) else (v,))]
    return out + [t for t in (encoder.last, encoder.slopes) if t is not None]


@pytest.mark.parametrize("norm", ["layer", "rms"])
def test_an_encoder_in_8_bits_shares_nothing_with_its_source(norm):
    enc = _encoder(norm, slopes=torch.tensor([0.5, 0.25]))
    for t in _tensors(enc)[:-1]:
        t.requires_grad_(True)
    enc8 = enc.in_8_bits()
    before = [t.clone() for t in _tensors(enc8)]
    theirs = {t.data_ptr() for t in _tensors(enc)}
    assert not any(t.requires_grad or t.data_ptr() in theirs for t in _tensors(enc8))
    with torch.no_grad():
        for t in _tensors(enc):
            t.mul_(3).add_(1)
    assert all(torch.equal(a, b) for a, b in zip(_tensors(enc8), before))


class DenseWeights(Weights):
    def quantize8(self, x, gelu=False):
        if x.stride(1) != 1:
            raise ValueError("x: want rows that are dense along the width")
        return super().quantize8(x, gelu)


def test_weights_of_any_strides():
    """Views that an encoder's plain products take: transposed, and one row for all channels."""
    enc = _encoder("layer")
    enc.he = DenseWeights()
    want = enc.in_8_bits().layers[0]["up"]
    enc.layers[0]["up"] = enc.layers[0]["up"].t().contiguous().t()
    enc.layers[1]["out"] = enc.layers[1]["out"][:1].expand(16, -1)
    enc8 = enc.in_8_bits()
    assert all(torch.equal(a, b) for a, b in zip(enc8.layers[0]["up"], want))
    assert (enc8.layers[1]["out"][0] == enc8.layers[1]["out"][0][:1]).all()


def _layer(width, inner):
    """A layer of one column to a head and one key head; what is not a product's weight does not matter here."""
    w = {n: torch.ones(1) for n in SentenceEncoder.NAMES}
    return {**w, "qkv": torch.ones(4, width), "out": torch.ones(width, 2), "up": torch.ones(inner, width), "down": torch.ones(width, inner)}


@pytest.mark.parametrize("width,inner,text", [(16, 16385, "layer 1: down has rows of 16385"), (16386, 24, "layer 1: qkv has rows of 16386")])
def test_rows_wider_than_8_bit_rows_are_refused_by_name(width, inner, text):
    """An encoder of plain products takes any width; rows in 8 bits are made up to 16384."""
    enc = SentenceEncoder(Weights(), [_layer(16, 16384), _layer(width, inner)], 2, kv_heads=1)
    with pytest.raises(ValueError, match=text + ".*16384"):
        enc.in_8_bits()
    SentenceEncoder(Weights(), [_layer(16, 16384), _layer(16384, 24)], 2, kv_heads=1).in_8_bits()
