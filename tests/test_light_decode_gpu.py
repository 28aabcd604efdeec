"""The light decode step as a user runs it: 4-bit weights, selected blocks and choice under rules on one decoder, against the oracle
on the weights that the 4-bit codes stand for."""
from dataclasses import replace

import numpy as np
import pytest
import torch

import oracle
import paper_2406_00059_amd as ld
from paper_2406_00059_amd.light import LightDecoder
from workloads import TINY, make_weights
from workloads.configs import weights_to
from helpers import prompt, rel_err

pytestmark = pytest.mark.gpu


def _stands_for(m, group, zeros, scales):
    """The matrix that ldk_linear_w4 multiplies with, column by column."""
    w = ld.W4Matrix.quantize(m.cuda(), group, 1, scales, zeros)
    eye = torch.eye(w.K, device="cuda")
    y = torch.empty(w.K, w.N, device="cuda")
    ld.ldk_linear_w4(w, eye, y, scratch=torch.empty(ld.ldk_linear_w4_scratch_bytes(w.K, w.N, w.K), dtype=torch.uint8, device="cuda"))
    return y.t().contiguous().cpu()


def _light(shape, seed, n_blocks=40, max_seqs=3, max_blocks=30, **kw):
    w = make_weights(shape, seed)
    model = ld.Model(shape, weights_to(w, "cuda"))
    kv = ld.KV(model, n_blocks, 64, max_seqs, max_blocks)
    kv.pool.fill_(float("nan"))
    return w, LightDecoder(model, kv, **kw)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("rows", [7, 256])
def test_light_decoder_matches_the_oracle_on_the_quantised_weights(zeros, rows):
    """fp32 decoder, budget beyond the context: logits within 1e-4 of the oracle's and the same greedy tokens, prompts in chunks or whole, with an
    observation appended behind the pending token."""
    w, light = _light(TINY, 5, group=32, zeros=zeros, budget=64, max_rows=rows)
    q = dict(w)
    for k in ("wqkv", "wo", "wgate_up", "wdown"):
        q[k] = [_stands_for(m, 32, zeros, torch.float32) for m in w[k]]
    q["lm_head"] = _stands_for(w["lm_head"], 32, zeros, torch.float32)
    okv = oracle.KV(oracle.Model(TINY, q), 40, 3, 30)
    rc, so = okv.alloc(0)
    seq = ld.ld_kv_alloc(light.kv.h)
    errs, ours, theirs = [], [], []
    for feed in (prompt(5, 1, 45, TINY.vocab), prompt(5, 2, 13, TINY.vocab)):
        rc, t, lg = okv.prefill(so, feed)
        theirs.append(t); ours.append(light.prefill(seq, feed)); errs.append(rel_err(light.logits[0].cpu(), lg))
        for _ in range(20):
            rc, t, lg = okv.decode(so)
            theirs.append(t); ours += light.step([seq]); errs.append(rel_err(light.logits[0].cpu(), lg))
    assert max(errs) <= 1e-4, max(errs)
    assert ours == theirs
    assert okv.block_table(so)[1].tolist() == ld.ld_kv_block_table(light.kv.h, seq).tolist()


@pytest.mark.parametrize("shape", [replace(TINY, dtype="bf16", n_heads=4, n_kv_heads=2, head_dim=128, name="tiny-bf16-hd128-gqa"),
                                   replace(TINY, dtype="bf16", window=50, name="tiny-bf16-band")])
def test_light_decoder_with_a_small_budget(shape):
    """Long contexts, few blocks: a batch's rows do not depend on each other, a mask is kept, and a refreshed fork goes on as its parent does."""
    _, light = _light(shape, 9, n_blocks=80, group=64, budget=5, keep_first=1, keep_last=2, penalties=(1.3, 0.2, 0.1))
    a, b = ld.ld_kv_alloc(light.kv.h), ld.ld_kv_alloc(light.kv.h)
    pa, pb = prompt(9, 1, 301, shape.vocab), prompt(9, 2, 90, shape.vocab)
    first = [light.prefill(a, pa), light.prefill(b, pb)]
    both = [light.step([a, b]) for _ in range(20)]
    assert (light.sel[0, 0] >= 0).sum() == min(5, len(range(max(0, 321 - shape.window) // 16 if shape.window else 0, 21)))
    # each alone, from the start, gives the same tokens
    for i, (s, p) in enumerate(((a, pa), (b, pb))):
        ld.ld_kv_free(light.kv.h, s)
        s2 = ld.ld_kv_alloc(light.kv.h)
        assert s2 == s and light.prefill(s2, p) == first[i]
        assert [light.step([s2])[0] for _ in range(20)] == [t[i] for t in both]
    child = ld.ld_kv_fork(light.kv.h, a, ld.ld_kv_len(light.kv.h, a))
    hist = light.history[a, :light.length[a]].tolist()
    keep = light.bounds.clone(), light.unit.clone()
    light.refresh(child, hist[:-1], hist[-1])
    blocks = torch.as_tensor(ld.ld_kv_block_table(light.kv.h, a)[:-1], device="cuda").long()      # all but the copied last one are shared
    assert torch.equal(light.bounds[:, blocks], keep[0][:, blocks]) and torch.equal(light.unit[:, blocks], keep[1][:, blocks])
    light.prompt[child] = light.prompt[a]
    mask = torch.zeros((1, shape.vocab // 32), dtype=torch.int32, device="cuda")
    mask[0, 3] = 0x00F00001
    allowed = {96, 116, 117, 118, 119}
    for _ in range(10):
        x, y = light.step([a], mask=mask)[0], light.step([child], mask=mask)[0]
        assert x == y and x in allowed
    mask[0, 3] = 0
    assert light.step([a], mask=mask) == [-1]


def test_light_decoder_refusals():
    _, light = _light(TINY, 3, group=64, max_rows=2)
    s = [ld.ld_kv_alloc(light.kv.h) for _ in range(3)]
    for bad in ([], [s[0], s[0]], s, [s[1]]):
        with pytest.raises(ValueError):
            light.step(bad)
    with pytest.raises(ValueError):
        light.prefill(s[0], [])
    light.prefill(s[0], [1, 2, 3])
    with pytest.raises(ValueError):
        light.refresh(s[0], [1, 2])
