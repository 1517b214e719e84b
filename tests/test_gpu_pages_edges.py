"""Attention over pages at the borders of its rules and with what its header allows and no ordinary call does, against its definition in float64.  How far
it may be off is derived in `paged.Batch.attention`."""
import pytest

from tests import test_gpu_pages as pages_tests
from tests.paged import Batch
from tests.test_gpu_pages import oqm  # noqa: F401

pytestmark = pytest.mark.gpu


def two_parts(b):
    """Whether the header promises probabilities in two 16-bit parts: up to 16 query rows of a KV head on average, not rounded."""
    return b.T * b.repeat <= 16 * b.B


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("repeat,extra", [(9, 1), (9, 37), (15, 3), (16, 0), (1, 720), (7, 61)])
def test_two_parts_up_to_the_average_that_the_header_names(oqm, dtype, repeat, extra):  # noqa: F811
    """48 sequences with a token each, and some tokens more anywhere in the batch."""
    new = [1 + extra // 48 + (1 if i < extra % 48 else 0) for i in range(48)]
    b = Batch(dtype=dtype, rows=[(13 * i) % 90 for i in range(48)], new=new, heads=1, repeat=repeat, d=64, layers=1, layer=0)
    assert two_parts(b)
    got = pages_tests.call(oqm, b, b.pages(oqm))
    pages_tests.close(b, got, b.attention(None, True, b.d ** -0.5, 0.0, None, one_part=False))
