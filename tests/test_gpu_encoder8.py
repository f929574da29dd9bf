"""Encoders in 8 bits on the GPU, beside the encoders that they come from."""
import numpy as np
import pytest
import torch

import paper_2210_02574_amd as pkg
import workloads as wl
from paper_2210_02574_amd.embedding import SentenceEncoder

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def he():
    assert torch.cuda.is_available(), "this test needs the MI355X"
    return pkg.HE.from_params(wl.C1B, device=0)


def rand(seed, *shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(dtype).cuda()


def offsets_of(lengths):
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]).tolist(), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("norm,pool,slopes", [("layer", "mean", True), ("layer", "first", False), ("rms", "mean", True), ("rms", "first", False)])
def test_later_changes_of_the_source_do_not_reach_an_encoder_in_8_bits(he, norm, pool, slopes):
    """All weights change in place, as a step of an optimizer changes them: the result stays bit for bit, and a second encoder made now has another one."""
    layers = [SentenceEncoder.random_layer(64, 2, 96, 5 + i, torch.float32, "cuda", std=0.1) for i in range(2)]
    last = 1 + rand(3, 64, scale=0.1) if norm == "rms" else None
    slopes = torch.tensor([0.5, 0.25], device="cuda") if slopes else None
    states, off = rand(1, 60, 64), offsets_of([20, 0, 1, 39])
    enc = SentenceEncoder(he, layers, 2, pool=pool, norm=norm, last=last, slopes=slopes)
    enc8 = enc.in_8_bits()
    before = enc8(states, off).clone()
    leaves = [v for w in layers for v in w.values()] + [t for t in (last, slopes) if t is not None]
    for i, t in enumerate(leaves):
        t.add_(rand(20 + i, *t.shape, scale=0.05).abs())
    assert torch.equal(enc8(states, off), before)
    assert not torch.equal(enc.in_8_bits()(states, off)[0], before[0])


def test_weights_of_any_strides(he):
    """Transposed views as plain products take them: the same encoder in 8 bits as with dense weights."""
    w = SentenceEncoder.random_layer(64, 2, 96, 5, torch.bfloat16, "cuda", std=0.1)
    states, off = rand(1, 60, 64, dtype=torch.bfloat16), offsets_of([20, 0, 1, 39])
    want = SentenceEncoder(he, [w], 2).in_8_bits()(states, off)
    views = {n: t.t().contiguous().t() if t.dim() == 2 else torch.stack([t, t], 1)[:, 0] for n, t in w.items() if "norm" not in n}
    enc = SentenceEncoder(he, [{**w, **views}], 2)
    enc(states, off)
    assert torch.equal(enc.in_8_bits()(states, off), want)


@pytest.mark.parametrize("norm", ["layer", "rms"])
def test_weights_of_an_encoder_in_8_bits_can_be_saved(he, norm, tmp_path):
    """torch.save takes no two types of tensors in one storage, as the integers and scales of HE.quantize8 are."""
    layers = [SentenceEncoder.random_layer(64, 2, 96, 5 + i, torch.bfloat16, "cuda", std=0.1) for i in range(2)]
    enc8 = SentenceEncoder(he, layers, 2, norm=norm, last=rand(3, 64, dtype=torch.bfloat16) if norm == "rms" else None).in_8_bits()
    states, off = rand(1, 60, 64, dtype=torch.bfloat16), offsets_of([20, 0, 1, 39])
    want = enc8(states, off)
    torch.save({"layers": enc8.layers, "last": enc8.last}, tmp_path / "weights")
    saved = torch.load(tmp_path / "weights", weights_only=True)
    enc8.layers, enc8.last = saved["layers"], saved["last"]
    assert torch.equal(enc8(states, off), want)
    x8, scale = he.quantize8(states)
    torch.save((x8, scale.clone()), tmp_path / "rows")
    assert all(torch.equal(a, b) for a, b in zip(torch.load(tmp_path / "rows", weights_only=True), (x8, scale)))
