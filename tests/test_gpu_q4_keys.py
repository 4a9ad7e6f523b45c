"""Keys of the cache held in 4 bits that are not finite, among a call's own tokens: exactly the rows that see them are NaN, on
either attention kernel."""
import numpy as np
import pytest

from layer_util import f64
from oracle import layer_oracle as L
from paper_2404_01365_b200 import binding as G
from q4_util import BatchQ4

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 2, 64), (16, 2, 112), (16, 1, 128), (6, 2, 256)])
@pytest.mark.parametrize("n,own,prefix", [(5, 9, 0), (40, 40, 0), (70, 300, 40), (300, 310, 20)])
@pytest.mark.parametrize("room", [1, 60000])      # keys that the table could hold beyond the sequence: what chooses the kernel
def test_a_key_that_some_rows_see(dtype, hq, hkv, hd, n, own, prefix, room):
    for back in {1, n // 2, n - 1}:
        b = BatchQ4([n, 1], [own, 30], prefix, hq, hkv, hd, 16, dtype, fill=0.0, seed=back, table_extra=-(-room // 16))
        at = own - back
        b.k_host[int(b.page_table[0, at // 16]), hkv - 1, at % 16, hd - 3] = NAN
        b.requantise()
        rows = {0, n - back - 1, n - back, n - 1, n} - {-1}
        want, mass = b.reference(rows)
        b.to_device()
        got = f64(b.attend())
        bad = np.zeros(got.shape[:2], bool)
        for t, s, i in L.places(b.q_start.numpy(), b.seq_len.numpy()):
            bad[t, -(hq // hkv):] = s == 0 and i >= at
        assert np.array_equal(np.isnan(got).all(2), bad) and np.array_equal(np.isnan(got).any(2), bad)
        bound = b.bound(want, mass)
        for t in rows:
            fine = ~bad[t]
            assert np.all(np.abs(got[t] - want[t])[fine] <= bound[t][fine])
        assert G.griffin_check_device_status(b.ws) == G.OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", [(1, 1, 80), (3, 1, 112), (5, 1, 208), (7, 1, 176)])
@pytest.mark.parametrize("n,own", [(1, 5000), (3, 3000), (6, 4000), (20, 1500), (40, 900)])
def test_clusters_of_widths_and_rows_that_fill_no_warp(dtype, hq, hkv, hd, n, own):
    # jobs that clusters of 8, 4, 2 CTAs take whole (by what the table holds), whose results end inside a warp's entries
    b = BatchQ4([1] * n, [own - 3 * i for i in range(n)], 0, hq, hkv, hd, 64, dtype, table_extra=0)
    want, mass = b.reference({0, n - 1})
    b.to_device()
    out = b.attend()
    for _ in range(3):
        assert np.array_equal(f64(b.attend()), f64(out))
    got, bound = f64(out), b.bound(want, mass)
    for t in {0, n - 1}:
        assert np.all(np.abs(got[t] - want[t]) <= bound[t])
    assert G.griffin_check_device_status(b.ws) == G.OK
