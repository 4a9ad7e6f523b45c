"""A value that is not finite reaches every token that sees it, however small its weight: 0 times it is NaN.  The weights here
underflow, and the keys that have them are worked on in other places (prefix and own keys, CTAs, warps, groups of warps) than
those that carry the sum, so that it is the joining of the places' results which has to keep them."""
import pytest

from layer_util import Batch
from q4_util import BatchQ4
from test_gpu_attn_causal import check

pytestmark = pytest.mark.gpu
NAN = float("nan")


def far(b, positions, values):
    """These positions of sequence 0 (the prefix, then its own) get logits far below the others': 64 * (32 + 32) * hd^-1/2 is 256 at
    256 entries, and fp32 ends at e^-104.  values: positions whose value is NaN."""
    at = lambda i: (b.prefix_pages[i // b.page], i % b.page) if i < b.prefix else (b.page_table[0, (i - b.prefix) // b.page], (i - b.prefix) % b.page)
    b.q[..., 0] = 64.0
    b.k_host[..., 0] = 32.0
    for i in positions:
        page, o = at(i)
        b.k_host[int(page), :, o, 0] = -32.0
    for i in values:
        page, o = at(i)
        b.v_host[int(page), b.hkv - 1, o, b.hd - 3] = NAN
    b.kmax = 32.0
    if isinstance(b, BatchQ4):
        b.requantise()
    return b


@pytest.mark.parametrize("kind", [Batch, BatchQ4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_lens,seq_lens,prefix,n", [
    ([1], [700], 0, 350),                     # one sequence: warps, CTAs, clusters of them
    ([1], [5000], 0, 2500),
    ([1, 1], [40, 90], 300, 300),             # a prefix that is worked on by itself
    ([2, 1, 1], [300, 90, 1], 500, 650),
    ([1] * 30, [300 + i for i in range(30)], 0, 130),
    ([1] * 80, [150 + i % 9 for i in range(80)], 0, 70),      # more jobs than are taken whole
    ([5], [900], 64, 500),
    ([40], [1500], 0, 800),
    ([300], [1200], 0, 850),                  # blocks of several row tiles, cut
    ([60, 3], [700, 30], 200, 450),
])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 1, 128), (2, 2, 64), (3, 1, 80), (2, 1, 256)])
def test_values_of_little_weight(kind, dtype, q_lens, seq_lens, prefix, n, hq, hkv, hd):
    T, end = sum(q_lens), prefix + seq_lens[0]
    for positions in (range(n), range(n, end)):      # in front of the others, and behind them
        b = kind(q_lens, seq_lens, prefix, hq, hkv, hd, 16, dtype, fill=0.0)
        check(far(b, positions, [positions[len(positions) // 3], positions[len(positions) // 2]]), {0, q_lens[0] - 1, T - 1} if T > 8 else None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 9, 70, 200])
def test_values_of_little_weight_on_either_kernel(dtype, n):
    # (a wide table sends pieces of many rows to the tcgen05 kernel)
    for room in (1, 4000):
        b = BatchQ4([n, 1], [n + 500, 20], 150, 8, 1, 128, 16, dtype, fill=0.0, table_extra=room)
        check(far(b, range(400), [3, 149, 150, 399]), {0, n - 1, n})
