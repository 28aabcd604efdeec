"""The light decoder and the engine on one cache: sequences that go from one to the other and back, are swapped, or are fed beside each other."""
from dataclasses import replace

import numpy as np
import pytest
import torch

import paper_2406_00059_amd as ld
from paper_2406_00059_amd.light import LightDecoder
from workloads import TINY, make_weights
from workloads.configs import weights_to
from helpers import Tokens, prompt, rel_err

pytestmark = pytest.mark.gpu


def _light(shape, seed, n_blocks=40, max_seqs=3, max_blocks=30, **kw):
    model = ld.Model(shape, weights_to(make_weights(shape, seed), "cuda"))
    kv = ld.KV(model, n_blocks, 64, max_seqs, max_blocks)
    kv.pool.fill_(float("nan"))
    return LightDecoder(model, kv, **kw)


def test_sequences_go_to_the_engine_and_back():
    """Fed by the engine, taken over, stepped, handed back: the engine's step feeds the token that was chosen last, as a prefill of that token behind
    a fork of the same positions does.  A token that the engine holds back is not fed on the way here unless refresh is given it."""
    shape = TINY
    light = _light(shape, 11, group=64, budget=64)
    h, sink = light.kv.h, Tokens()
    s = ld.ld_kv_alloc(h)
    p = prompt(11, 1, 37, shape.vocab)
    ld.ld_prefill(h, s, p, callback=sink)
    light.refresh(s, p, sink.last()[0])
    hist = p.tolist() + sink.last()
    for _ in range(5):
        hist += light.step([s])
    fork = ld.ld_kv_fork(h, s, ld.ld_kv_len(h, s))
    _, want = ld.ld_prefill(h, fork, [hist[-1]], logits_vocab=shape.vocab)
    _, got = ld.ld_decode_step(h, [s], callback=sink, logits_vocab=shape.vocab)
    assert rel_err(got[0], want) <= 1e-5      # one row of one float32 path, in the kernels of a step and in those of a chunk
    hist += sink.last()
    light.refresh(s, hist[:-1], hist[-1])
    hist += light.step([s])
    assert light.history[s, :len(hist)].tolist() == hist and ld.ld_kv_len(h, s) == len(hist) - 1
    light.refresh(fork, hist[:-2])
    light.prefill(fork, hist[-2:-1])
    assert ld.ld_kv_len(h, fork) == len(hist) - 1
