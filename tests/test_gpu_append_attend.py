"""New keys and values that are attended over by the call right behind the one that writes them, again and again over the same
pages: what an attention call reads is what the append in front of it wrote, values that are not finite among it."""
import numpy as np
import pytest
import torch

from layer_util import Batch, f64
from oracle import layer_oracle as L
from paper_2404_01365_b200 import binding as G
from q4_util import BatchQ4

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("kind", [Batch, BatchQ4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 1, 128), (2, 2, 64), (2, 1, 256)])
@pytest.mark.parametrize("q_lens,own,prefix", [([3], 40, 0), ([40, 1], 60, 30), ([150], 300, 0)])
def test_values_that_change_from_call_to_call(kind, dtype, hq, hkv, hd, q_lens, own, prefix):
    b = kind(q_lens, [own] * len(q_lens), prefix, hq, hkv, hd, 16, dtype, fill=0.0).to_device()
    append = G.griffin_kv_append_q4 if kind is BatchQ4 else G.griffin_kv_append
    q, k = b.q.to(DEV), b.k.to(DEV)
    places = [(t, s, i) for t, s, i in L.places(b.q_start.numpy(), b.seq_len.numpy())]
    n = q_lens[0]
    values, outs = [], []
    for turn in range(8):
        v = b.v.clone()
        v[turn * n // 8, hkv - 1, hd - 1] = float("nan")      # a token of sequence 0, another one each time
        values.append(v.to(DEV))
    torch.cuda.synchronize()
    for v in values:
        append(b.desc, b.batch, b.cache, None, None, k, v, None, b.ws)
        outs.append(b.attend(q=q))
    assert G.griffin_check_device_status(b.ws) == G.OK
    for turn, out in enumerate(outs):
        nan = np.isnan(f64(out)[:, hq - 1, hd - 1])
        assert np.array_equal(nan, [s == 0 and t >= turn * n // 8 for t, s, i in places])
