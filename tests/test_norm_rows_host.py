"""What a row of the norm is: the binding refuses tensors that leave it open, the library widths that 32 bits do not count."""
import pytest

from paper_2105_01827_amd import binding
from tests.test_kv4_host import CODES, Context, _norm, _on_gpu, ctx  # noqa: F401


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


@pytest.mark.parametrize("width", [(1 << 30) + 1, (1 << 31) - 1024, (1 << 31) - 1])
def test_widths_beyond_32_bits_are_refused(ctx, width):  # noqa: F811
    """columns and groups are counted in 32 bits"""
    for more in (dict(), CODES, CODES | dict(how__group=128), dict(out__type=3, how__limit=63, how__scales=1 << 20)):
        strides = {f"{name}__stride": width for name in ("x", "add", "sum", "out")}
        assert _norm(ctx, width=width, **(strides | more)) == binding.GALA_EARG
        strides = {f"{name}__stride": 1 << 30 for name in ("x", "add", "sum", "out")}
        assert _norm(ctx, width=1 << 30, rows=0, **(strides | more)) != binding.GALA_EARG
