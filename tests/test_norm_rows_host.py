"""What a row of the norm is: the binding refuses tensors that leave it open."""
import pytest

from tests.test_kv4_host import Context, _on_gpu


@pytest.mark.parametrize("shape", [(2, 5, 8), (1, 5, 8), (5, 1, 8), (2, 3, 4, 5)])
def test_more_dimensions_are_refused(shape):
    for kwargs in (dict(), dict(weight=_on_gpu(shape[-1]))):
        with pytest.raises(ValueError, match="rows x width"):
            Context().rms_norm(_on_gpu(*shape), _on_gpu(*shape), **kwargs)


def test_other_tensors_may_have_heads():
    """a row of heads is a row of as many numbers"""
    for change in (dict(out=_on_gpu(5, 2, 4)), dict(add=_on_gpu(5, 4, 2)), dict(sum_out=_on_gpu(5, 1, 8))):
        with pytest.raises(AssertionError, match="gala_rms_norm was called"):
            Context().rms_norm(**(dict(x=_on_gpu(5, 8), out=_on_gpu(5, 8)) | change))
