"""What the Python binding refuses before a pointer is taken (no GPU: these are tensors of the host, which the
binding refuses last)."""
import pytest

from paper_2606_18954_amd import graphattn as G

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("name", ["MXFP4", "fp4", "bfloat16", "float32", "", None, 2])
def test_a_type_that_is_none_is_refused(name):
    """(Taken for another type, the kernels would read past a smaller pool's end.)"""
    with pytest.raises(ValueError, match="mxfp4"):
        G.make_params(4, 2, 64, 3, name)
