"""paged_attn_forward on prefills in which the new tokens are most or all of the keys, so that shares cut blocks among the tokens that see each other."""
import pytest

from tests.sampling_util import Paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,heads,dim,lens,new", [
    ("bf16", (16, 1), 64, [601], [601]), ("bf16", (28, 4), 128, [640, 333], [640, 300]), ("bf16", (300, 1), 64, [71], [71]),
    ("f32", (8, 2), 128, [520], [500]), ("f32", (14, 2), 64, [400, 65], [400, 64]), ("f32", (40, 1), 64, [130], [130]),
])
def test_prefill_from_nothing(dtype, heads, dim, lens, new):
    x = Paged(dtype, heads, dim, 16, lens, new, pad=2, seed=40)
    x.check(*x.attend())
