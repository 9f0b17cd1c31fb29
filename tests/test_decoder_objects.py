"""Cache and Rotary take their pointers once, so what they were made of is there to be read only (no GPU)."""
import ast
import inspect

import pytest
import torch

from paper_2203_00091_amd import Cache, Rotary, binding


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


def test_no_name_of_the_binding_is_taken_twice():
    """(A second definition takes the first one's place, in every call that needs it.)"""
    names = [n.name for n in ast.parse(inspect.getsource(binding)).body if isinstance(n, (ast.FunctionDef, ast.ClassDef))]
    assert len(names) == len(set(names))
