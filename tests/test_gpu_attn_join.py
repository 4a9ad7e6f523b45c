"""Blocks of rows that are cut, of calls with few blocks: how many rows a block has and how many blocks there are says how many
CTAs of the joining kernel take them, and which."""
import pytest

from layer_util import Batch
from q4_util import BatchQ4
from test_gpu_layer import check_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [Batch, BatchQ4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 256])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 1), (10, 5), (36, 36), (37, 37), (38, 38), (33, 11)])
def test_rows_and_blocks(kind, dtype, hd, hq, hkv):
    for n, own in ((1, 700), (2, 5), (7, 2100), (8, 300), (9, 300), (17, 1000), (65, 400), (129, 400)):
        if n * hq > 1300 or own * hkv > 40000:
            continue
        check_attention(kind([n], [own], 0, hq, hkv, hd, 32, dtype, table_extra=300), rows={0, n // 2, n - 1})


@pytest.mark.parametrize("kind", [Batch, BatchQ4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [80, 208])
def test_several_sequences(kind, dtype, hd):
    # cuts of several blocks, of different lengths, some of them of one sequence; and sequences that see nothing
    for q_lens, seq_lens in (([40, 3], [900, 40]), ([70, 0, 50], [70, 9, 3000]), ([30, 20, 25, 9], [500, 20, 700, 600]), ([150, 150], [150, 700]),
                             ([260], [250]), ([90, 40], [0, 400])):
        check_attention(kind(q_lens, seq_lens, 0, 4, 1, hd, 32, dtype, table_extra=300, extra_rows=1), rows={0, q_lens[0] - 1, sum(q_lens) - 1, sum(q_lens) // 2})
