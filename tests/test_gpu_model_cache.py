"""The quantised cache of a model as a caller sees it (GmModel.read_cache)."""
import numpy as np
import pytest
import torch

import synth

from test_gpu_parity import gpu_model, run

pytestmark = pytest.mark.gpu


def filled_model():
    cfg = synth.preset("tiny_decoder", batch=2)
    ids, mask = synth.make_inputs(cfg, 3, seq=12)
    m = gpu_model(cfg, synth.make_weights(cfg, 5), max_seq=cfg.seq, kv_cache=True, kv_bits=8)
    run(m, ids, mask)
    torch.cuda.synchronize()
    return m


def stream_of(t):
    """The stream whose memory a tensor lies in."""
    at = [g["stream"] for g in torch.cuda.memory_snapshot()
          if g["address"] <= t.data_ptr() < g["address"] + g["total_size"]]
    assert len(at) == 1
    return at[0]


def test_rows_read_on_another_stream_belong_to_it():
    m = filled_model()
    here = m.read_cache(0, 12)
    s = torch.cuda.Stream()
    there = m.read_cache(0, 12, stream=s)
    torch.cuda.synchronize()
    for a, b in zip(here, there):
        assert torch.equal(a, b) and a.abs().sum() > 0
        assert stream_of(b) == s.cuda_stream != stream_of(a)


def test_rows_past_the_cache_and_fewer_sequences():
    m = filled_model()
    k, v = m.read_cache(0, 12)
    for batch in (1, 0):
        for a, b in zip((k, v), m.read_cache(0, 12, batch=batch)):
            assert torch.equal(a[:batch], b)
    long = m.read_cache(0, 200)
    assert torch.equal(long[0][:, :12], k) and not long[0][:, m.c.max_seq:].any()
    assert np.isfinite(long[1].float().cpu().numpy()).all()
