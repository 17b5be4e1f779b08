"""What the binding takes for the tensors of a cache."""
import pytest
import torch

import paper_2301_11913_amd as sw


def tensors(cfg, scale):
    made = {n: torch.zeros(s, dtype=d) for n, (s, d) in cfg.shapes().items()}
    for n in ("k_scales", "v_scales"):
        made[n] = made[n].to(scale)
    return made


@pytest.mark.parametrize("scale", [torch.bfloat16, torch.int16, torch.uint16])
def test_16_bit_scales_are_bf16_values_or_their_bit_patterns(scale):
    cfg = sw.CacheConfig(4, 2, 64, 16, 3, 2, 5, "bf16", 16)
    assert sw.Cache(cfg, **tensors(cfg, scale)).c.k_scales


@pytest.mark.parametrize("bits,scale", [(16, torch.float16), (16, torch.float32), (32, torch.bfloat16), (32, torch.int32), (32, torch.float64)])
def test_scales_of_another_type_are_refused(bits, scale):
    """fp16 values have two bytes as well, but their bits mean other numbers."""
    cfg = sw.CacheConfig(4, 2, 64, 16, 3, 2, 5, "bf16", bits)
    with pytest.raises(TypeError, match="k_scales must be"):
        sw.Cache(cfg, **tensors(cfg, scale))


@pytest.mark.parametrize("name", ["k_codes", "v_codes"])
def test_codes_are_int8(name):
    cfg = sw.CacheConfig(4, 2, 64, 16, 3, 2, 5, "bf16", 16)
    made = tensors(cfg, torch.bfloat16)
    made[name] = made[name].to(torch.uint8)
    with pytest.raises(TypeError, match=name):
        sw.Cache(cfg, **made)
