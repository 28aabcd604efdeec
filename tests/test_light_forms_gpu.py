"""Forms of the light decode step's operators that sizes of a whole model take: workgroups with several units of outputs, gated products of one and
two rows, wide slices of the vocabulary, and the bf16 decoder against the oracle."""
from dataclasses import replace

import numpy as np
import pytest
import torch

import oracle
import paper_2406_00059_amd as ld
from paper_2406_00059_amd.light import LightDecoder
from workloads import TINY, gen, make_weights
from workloads.configs import weights_to
from helpers import prompt, rel_err
from test_light_decode_gpu import _stands_for
from test_light_ops_gpu import LINEAR, _adjust64, _choose, _linear, _packed, _rel, _rules, _w4

pytestmark = pytest.mark.gpu


def _gated(W, x, N):
    gu = x @ W.t()
    return gu[:, :N] * torch.sigmoid(gu[:, :N]) * gu[:, N:]


def _rows(seed, T, K):
    return gen.normal(seed, 5, (T, K)), gen.normal(seed, 6, (K,), std=0.1, mean=1.0)


def _normed(x, g):
    x = x.double()
    return x / torch.sqrt((x ** 2).mean(1, keepdim=True) + 1e-5) * g.double()


# The tolerances are those of the same products at other sizes: LINEAR for a product, three times it where two products and the activation meet.

@pytest.mark.parametrize("N,K,group,zeros", [(8224, 512, 128, True), (8232, 1024, 32, False), (11008, 256, 64, True), (24600, 128, 128, False)])
@pytest.mark.parametrize("T", [1, 2])
def test_w4_gated_rows_with_several_units_a_workgroup(T, N, K, group, zeros):
    c, s, z, W = _w4(N, 2 * N, K, group, zeros, torch.bfloat16)
    s, W = s * 0.125, W * 0.125
    x, g = _rows(N, T, K)
    y = _linear(_packed(c, s, z, N, K, group, 2), x, ld.LDK_SWIGLU, g)
    assert _rel(y, _gated(W, _normed(x, g), N)) <= 3 * LINEAR


@pytest.mark.parametrize("N,K,group,zeros", [(16400, 384, 128, False), (16411, 512, 32, True), (33000, 256, 64, False), (50001, 129, 128, True)])
@pytest.mark.parametrize("epilogue", [ld.LDK_STORE, ld.LDK_ADD])
@pytest.mark.parametrize("T", [1, 2])
def test_w4_plain_rows_with_several_units_a_workgroup(T, epilogue, N, K, group, zeros):
    c, s, z, W = _w4(N, N, K, group, zeros, torch.bfloat16)
    x, g = _rows(N, T, K)
    ref, y0 = _normed(x, g) @ W.t(), gen.normal(N, 7, (T, N))
    y = _linear(_packed(c, s, z, N, K, group), x, epilogue, g, y0.to("cuda") if epilogue == ld.LDK_ADD else None)
    if epilogue == ld.LDK_ADD:
        assert _rel(y.cpu().double() - y0.double(), ref) <= 2 * LINEAR
    else:
        assert _rel(y, ref) <= LINEAR


@pytest.mark.parametrize("K", [512, 5120, 6144, 11008, 14336])
@pytest.mark.parametrize("group,zeros,scales", [(32, True, torch.bfloat16), (64, False, torch.float32), (128, True, torch.float32), (128, False, torch.bfloat16)])
@pytest.mark.parametrize("T", [1, 2, 20, 300])
def test_w4_gated_products_of_every_group_and_length(T, group, zeros, scales, K):
    N = 88
    c, s, z, W = _w4(K + group, 2 * N, K, group, zeros, scales)
    s, W = s * 0.125, W * 0.125
    x, g = _rows(K, T, K)
    y = _linear(_packed(c, s, z, N, K, group, 2), x, ld.LDK_SWIGLU, g)
    assert _rel(y, _gated(W, _normed(x, g), N)) <= 3 * LINEAR


@pytest.mark.parametrize("R,V", [(33, 32000), (58, 32000), (70, 32003), (600, 5000), (1, 100001)])
def test_choose_with_slices_of_every_width(R, V):
    """From 33 rows of 32000 tokens on a slice has more tokens than its threads take at first; 58 rows take the widest ones."""
    logits = gen.normal(V + R, 20, (R, V), std=3.0)
    k = _rules(V + R, R, V, 300)
    k["mask"][:, : V // 64] |= -1 << 16
    tok, adj = _choose(logits, want=True, **k)
    rows = range(R) if R < 10 else [0, 1, R // 2, R - 1]
    for r in rows:
        one = dict(k, history=k["history"][r:r + 1], history_len=k["history_len"][r:r + 1], n_prompt=k["n_prompt"][r:r + 1],
                   penalties=k["penalties"][r:r + 1], bias_start=k["bias_start"][r:r + 2], mask_row=k["mask_row"][r:r + 1])
        ref = _adjust64(logits[r:r + 1], one)[0]
        gone = np.isinf(ref)
        assert (np.isinf(adj[r].numpy()) == gone).all()
        size = np.abs(logits[r].numpy()).max() * 2 + 60 + 12      # as in the test of few rows: four roundings
        assert np.abs(adj[r].numpy()[~gone] - ref[~gone]).max() <= 4 * 2.0 ** -24 * size
    assert torch.equal(tok.long(), adj.argmax(1))      # the first of the largest
    temp, seed, pos = torch.full((R,), 0.8), torch.arange(R) * 977 + 5, torch.arange(R, dtype=torch.int32)
    out = torch.empty(R, dtype=torch.int32, device="cuda")
    ld.ldk_sample(adj.cuda(), temp.cuda(), seed.cuda(), pos.cuda(), out)
    assert torch.equal(_choose(logits, temperature=temp, seed=seed, pos=pos, **k)[0], out.cpu())


@pytest.mark.parametrize("shape", [replace(TINY, dtype="bf16", n_heads=4, n_kv_heads=2, head_dim=128, name="tiny-bf16-hd128-gqa"),
                                   replace(TINY, dtype="bf16", n_heads=8, n_kv_heads=1, head_dim=128, window=60, name="tiny-bf16-hd128-mqa-band"),
                                   replace(TINY, dtype="bf16", name="tiny-bf16-hd64")])
def test_light_decoder_on_bf16_matches_the_oracle(shape):
    """Budget beyond the context: prompt in chunks through the chunk attention (128 dimensions) and steps through the matrix-core attention, logits
    against the oracle on the matrices that the codes stand for, tokens given by masks of one token.  2e-2: what the engine's bf16 path is held to
    (a key or value on the edge between two bf16 numbers may round either way)."""
    w = make_weights(shape, 17)
    model = ld.Model(shape, weights_to(w, "cuda"))
    kv = ld.KV(model, 40, 64, 2, 20)
    kv.pool.fill_(float("nan"))
    light = LightDecoder(model, kv, group=64, budget=64, max_rows=48)
    q = {k: [m.float() for m in v] if isinstance(v, list) else v.float() for k, v in w.items()}
    for k in ("wqkv", "wo", "wgate_up", "wdown"):
        q[k] = [_stands_for(m, 64, False, torch.bfloat16) for m in w[k]]
    q["lm_head"] = _stands_for(w["lm_head"], 64, False, torch.bfloat16)
    okv = oracle.KV(oracle.Model(replace(shape, dtype="f32"), q, kv_round=1), 40, 2, 20)
    rc, so = okv.alloc(0)
    seq = ld.ld_kv_alloc(kv.h)
    forced, errs = prompt(17, 3, 30, shape.vocab).tolist(), []
    empty = np.zeros((0, shape.n_layers, 2, shape.n_kv_heads, shape.head_dim))

    def only(t):
        m = torch.zeros((1, shape.vocab // 32), dtype=torch.int32)
        m[0, t // 32] = int(np.uint32(1 << (t % 32)).view(np.int32))
        return m.cuda()

    def chosen(t, lg):
        errs.append(rel_err(light.logits[0].cpu(), lg))
        assert okv.inject(so, empty, pending=t) == 0

    for feed, n in ((prompt(17, 1, 130, shape.vocab), 15), (prompt(17, 2, 21, shape.vocab), 15)):
        t = forced.pop()
        assert light.prefill(seq, feed, mask=only(t)) == t
        chosen(t, okv.prefill(so, feed)[2])
        for _ in range(n - 1):
            t = forced.pop()
            assert light.step([seq], mask=only(t)) == [t]
            chosen(t, okv.decode(so)[2])
    assert max(errs) <= 2e-2, max(errs)
    assert okv.length(so) == ld.ld_kv_len(kv.h, seq)
