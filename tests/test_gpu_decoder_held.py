"""What the decoder's cache in 4 bits holds after steps that ran as a graph, whose lengths only the device counts."""
import pytest
import torch

from paper_2404_01365_b200 import binding as G
from paper_2404_01365_b200.decoder import Decoder, DecoderConfig, random_weights

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_held_after_replayed_steps(dtype):
    cfg = DecoderConfig(vocab=96, d=256, n_layers=2, n_q_heads=4, n_kv_heads=2, head_dim=64, d_ff=512, dtype=dtype, page_size=8, cache="q4")
    n_seq, steps = 3, 11
    dec = Decoder(cfg, random_weights(cfg, device=DEV), 32, n_seq, 16, keep=0.5, device=DEV)
    tokens = torch.randint(0, cfg.vocab, (20 + steps * n_seq,), generator=torch.Generator().manual_seed(2)).to(DEV)
    new = tokens[20:].view(steps, n_seq)
    dec.prompt(tokens[:20])
    for t in range(steps):
        dec.step(new[t])
    want = [dec.held(i) for i in range(cfg.n_layers)]

    dec.restart()
    at = new[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dec.step(at)
    assert dec.held(0)[1][0].shape == (n_seq, 0, 2, 64)       # captured, not run
    for t in range(steps):
        at.copy_(new[t])
        graph.replay()
        assert dec.held(0)[1][0].shape == (n_seq, t + 1, 2, 64)
    for i in range(cfg.n_layers):
        for a, b in zip(want[i], dec.held(i)):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert dec.status() == G.OK
