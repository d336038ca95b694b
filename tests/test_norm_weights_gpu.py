"""symar.Norm goes by its tensors as they are when it is called: a program may have given them other memory, another type or another size since (weights that are
loaded or cast in place, Module.half() among them)."""
import pytest
import torch

from paper_2607_16100_b200 import symar

pytestmark = pytest.mark.gpu


def normal(*shape, seed, dtype=torch.bfloat16):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("which", ["weight", "bias"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_memory_of_another_kind(which, dtype):
    x = normal(5, 256, seed=1)
    t = normal(256, seed=2)
    kept = t.data                                                    # (the old memory stays, so that nobody's is read either way)
    norm = symar.Norm("rms", **{which: t})
    first = symar.norm(x, before=norm)[0]
    t.data = normal(256, seed=3, dtype=dtype)
    got = symar.norm(x, before=norm)[0]
    assert torch.equal(got, symar.norm(x, before=symar.Norm("rms", **{which: normal(256, seed=3, dtype=dtype)}))[0]) and not torch.equal(got, first)
    t.data = kept
    assert torch.equal(symar.norm(x, before=norm)[0], first)
    t.add_(1)                                                        # in place
    assert torch.equal(symar.norm(x, before=norm)[0], symar.norm(x, before=symar.Norm("rms", **{which: t.clone()}))[0])


def test_a_module_that_is_cast():
    x = normal(4, 128, seed=1)
    layer = torch.nn.LayerNorm(128, device="cuda")
    with torch.no_grad():
        layer.weight.copy_(normal(128, seed=2)), layer.bias.copy_(normal(128, seed=3))
    kept = layer.weight.data, layer.bias.data
    norm = symar.Norm("layer", layer.weight, layer.bias, eps=layer.eps)
    want = symar.norm(x, before=norm)[0]
    layer.bfloat16()
    assert torch.equal(symar.norm(x, before=norm)[0], want)          # (the values are bf16's)
    with pytest.raises(symar.SymarError) as e:
        layer.half()
        symar.norm(x, before=norm)
    assert e.value.code == symar.ERR_UNSUPPORTED
    del kept


def test_memory_that_does_not_fit_is_refused():
    x = normal(3, 64, seed=1)
    w, b = normal(64, seed=2), normal(64, seed=3)
    kept = w.data, b.data
    norm = symar.Norm("rms", w, b)
    symar.norm(x, before=norm)
    for t in (w, b):
        was = t.data
        for other in (normal(32, seed=4), normal(128, seed=4)[::2], normal(1, 64, seed=4), t.data.float(), t.data.cpu()):
            try:
                t.data = other
            except RuntimeError:
                continue
            with pytest.raises(symar.SymarError):
                symar.norm(x, before=norm)
        t.data = was
        symar.norm(x, before=norm)
    norm.weight = normal(64, seed=5)
    assert torch.equal(symar.norm(x, before=norm)[0], symar.norm(x, before=symar.Norm("rms", normal(64, seed=5), b))[0])
    del kept
