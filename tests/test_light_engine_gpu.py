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


@pytest.mark.parametrize("shape", [TINY, replace(TINY, dtype="bf16", n_heads=4, n_kv_heads=2, head_dim=128, name="tiny-bf16-hd128-gqa")],
                         ids=["f32", "bf16-gqa"])
def test_a_swapped_sequence_goes_on_as_an_undisturbed_one(shape):
    """Swapped out, its blocks taken and described by another sequence, swapped in on other blocks and on the same ones: refused until it is
    refreshed, then token for token what a decoder without the swap gives."""
    light = _light(shape, 13, n_blocks=60, group=64, budget=5, keep_last=2)
    h, p = light.kv.h, prompt(13, 1, 150, shape.vocab)
    s = ld.ld_kv_alloc(h)
    want = [light.prefill(s, p)] + [light.step([s])[0] for _ in range(30)]
    ld.ld_kv_free(h, s)
    assert ld.ld_kv_alloc(h) == s
    got = [light.prefill(s, p)] + [light.step([s])[0] for _ in range(10)]
    for keep in (True, False):      # the other sequence keeps the blocks, or has freed them again
        buf = torch.empty(ld.ld_kv_swap_bytes(h, s), dtype=torch.uint8, pin_memory=True)
        ld.ld_kv_swap_out(h, s, buf)
        other = ld.ld_kv_alloc(h)
        light.prefill(other, prompt(13, 2, 170, shape.vocab))
        if not keep:
            ld.ld_kv_free(h, other)
        old = light.table[s].tolist()
        ld.ld_kv_swap_in(h, s, buf)
        torch.cuda.synchronize()
        n = ld.ld_kv_len(h, s)
        with pytest.raises(ValueError):
            light.step([s])
        assert ld.ld_kv_len(h, s) == n
        hist = p.tolist() + got
        light.refresh(s, hist[:-1], hist[-1])
        assert (light.table[s].tolist() != old) == keep
        got += [light.step([s])[0] for _ in range(10)]
    assert got == want
