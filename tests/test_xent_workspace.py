"""The loss's workspace (no GPU needed): one for more tokens, more features or a larger vocabulary is never smaller, so it holds whatever a
smaller problem's own would, and gives the same results."""
import random

import pytest

from paper_2502_02406_amd import binding as B
from test_abi import lib  # noqa: F401

SIZE = B.lvx_xent_workspace_bytes


@pytest.mark.parametrize("dtype", [B.LVX_BF16, B.LVX_F32])
def test_more_never_takes_less(lib, dtype):  # noqa: F811
    # where a piece of the vocabulary ends and a second one begins, and where rows of the logits' gradient get longer
    for n, E in ((4096, 1024), (4097, 512), (2048, 4096), (16384, 64)):
        sizes = [SIZE(n, E, V, dtype) for V in (1, 256, 8192, 8193, 65536, 65537, 131072, 131073, 200000, 262144, 262145, 1 << 20)]
        assert sizes == sorted(sizes), (n, E)
    for E, V in ((512, 131072), (64, 1000), (1024, 50021), (4096, 300), (128, 1 << 20)):
        sizes = [SIZE(n, E, V, dtype) for n in (1, 32, 33, 64, 65, 128, 129, 256, 257, 511, 512, 1000, 2048, 4096, 4097, 5000, 16384, 16385, 100000)]
        assert sizes == sorted(sizes), (E, V)
    rng = random.Random(1)
    log = lambda top: int(round(2.0 ** rng.uniform(0.0, top)))
    for _ in range(20000):
        n, E, V = log(17), 64 * log(7), log(19)
        n2, E2, V2 = (rng.choice((k, max(1, k - rng.randrange(300)), max(1, k // rng.choice((2, 3, 7))), rng.randint(1, k))) for k in (n, E // 64, V))
        assert SIZE(n2, 64 * E2, V2, dtype) <= SIZE(n, E, V, dtype), ((n2, 64 * E2, V2), (n, E, V))


@pytest.mark.parametrize("dtype,el", [(B.LVX_BF16, 2), (B.LVX_F32, 4)])
def test_what_it_takes_stays_bounded(lib, dtype, el):  # noqa: F811
    """A piece of the logits' gradient is a GiB, or 8192 entries of the vocabulary where these are more; beside it, what goes by the tokens and the
    features: their list, the statistics, and the sums of dx and dw in float32."""
    for n, E, V in ((4096, 4096, 131072), (4096, 1024, 131073), (100000, 64, 50000), (16, 4096, 32768), (300, 512, 5003), (1, 64, 1)):
        rows = (n + 255) // 256 * 256
        piece = min((V + 255) // 256 * 256 * rows * el, max(1 << 30, 8192 * rows * el))
        beside = 64 * rows * el + 16 * rows * (V // 64 + 8) + 4 * (rows * (E + 256) + 512 * 256 * 256) + (32 << 20) + 4096
        assert SIZE(n, E, V, dtype) <= piece + beside, (n, E, V)
