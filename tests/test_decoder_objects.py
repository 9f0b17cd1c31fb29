"""Cache and Rotary take their pointers once, so what they were made of is there to be read only (no GPU)."""
import pytest
import torch

from paper_2203_00091_amd import Cache, Rotary


@pytest.mark.parametrize("kind, names", [(Cache, "k v k_scale v_scale table len B Hk d device"), (Rotary, "cos sin pos interleaved device")])
def test_the_tensors_cannot_be_exchanged(kind, names):
    o, t = object.__new__(kind), torch.zeros(3)
    for name in names.split():
        with pytest.raises(AttributeError):
            setattr(o, name, t)
        setattr(o, "_" + name, t)
        assert getattr(o, name) is t
        with pytest.raises(AttributeError):
            delattr(o, name)
    with pytest.raises(AttributeError):
        o.page = 16
