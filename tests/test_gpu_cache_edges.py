"""The paged cache on the GPU: what lies outside the requests' tokens, bounds far above them, and the
forms of slots and writes that large calls take."""
import numpy as np
import pytest
import torch

from paper_2608_26806_gb300 import avtp
from tests.cache_util import Batch
from tests.gpu_util import ensure_built

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    ensure_built()


def status(call):
    return avtp.read_device_status(call.workspace)


# ---------------------------------------------------------------- attention
@pytest.mark.parametrize("Hq,Hkv,d", [(8, 8, 128), (16, 16, 64), (20, 4, 128)])
def test_slots_behind_a_requests_last_token_change_no_bit(Hq, Hkv, d):
    """The keys' rows that follow a request's last token in its page, as zeros, NaN and infinities. A key
    near the end stands out by 2^8 to 2^13 weights: far enough that a row's reference may move for it, not so
    far that its own sum makes it."""
    b = Batch([(164 + r % 9, 1) for r in range(60)], Hq, Hkv, d, 64, seed=d)
    G = Hq // Hkv
    for r, (s, _) in enumerate(b.requests):
        q = b.q[r].float().view(Hkv, G, d)[:, 0]
        key = (9.0 * d ** 0.5 * q / (q * q).sum(-1, keepdim=True)).to(torch.bfloat16)
        b.rows[r][0][s - 2] = key
        b.cache.k[int(b.table[r, (s - 2) // 64]), (s - 2) % 64] = key.cuda()
    spare = torch.isnan(b.cache.k)
    got = []
    for fill in (0.0, float("nan"), float("inf"), -3e38):
        b.cache.k[spare] = fill
        c = b.call().run()
        assert status(c) == avtp.OK
        b.check(c.o, c.lse)
        got.append((c.o, c.lse))
    for o, lse in got[1:]:
        assert torch.equal(o, got[0][0]) and torch.equal(lse, got[0][1])
