"""paged_attn_forward where some of a call's sequences have no new tokens, as in a captured step whose rollouts end one by one: they have no tokens, or no page, or both,
and the others' results do not change."""
import numpy as np
import pytest

from tests.sampling_util import Paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,heads,dim,shared", [("bf16", (28, 4), 128, 640), ("bf16", (14, 2), 64, 64), ("f32", (8, 2), 64, 320)])
@pytest.mark.parametrize("idle", [[0], [0, 1, 2], [3], [0, 2, 4]])
def test_idle_sequences_beside_shared_pages(dtype, heads, dim, shared, idle):
    """The shared pages are found through the first sequence that has new tokens: an idle one's row of the table may hold anything."""
    lens = [shared + 5 + 37 * i for i in range(5)]
    new = [0 if i in idle else 1 + i % 2 for i in range(5)]
    x = Paged(dtype, heads, dim, 32, lens, new, shared, pad=2, seed=50)
    for i in idle:
        x.lens[i] = 0 if i % 2 else -3
        x.table[i] = -1 if i % 2 else x.pages + 7
    want = x.oracle()
    x.check(*x.attend(), want)
    x.check(*x.attend(shared_len=shared), want)
    assert (np.diff(x.cu)[idle] == 0).all()
