"""The operators of a decode step that reads few bytes, as cases to time and to compare.

Four operators, each in its plain form (elementary torch operations in float32) and through the package's entry points:

  linear   a linear layer on 4-bit weights with a scale (and, where the checkpoint has them, a zero point) per group of
           input columns, with the RMSNorm ahead of it and SwiGLU behind it where a layer has them.
  summary  the 8-bit bounds of the keys of each 16-position block of the paged cache, brought up to date after an append.
  sparse   decode attention over the cache blocks that those bounds select for each query.
  choose   penalties for repeated tokens, biases and grammar masks on logits, and the token's choice.

Shapes are the repository's own decoder shapes; batch sizes, contexts and chunk lengths are those of its workloads (one
sequence at a context of some 1500 tokens, 32 sequences U[512, 8192], observations of 256 tokens behind their pending
token, the mixed step of 1056 rows).  Block tables are seeded permutations of the pool.
"""
import math

import numpy as np
import torch

from workloads import LLAMA7B, LLAMA13B, MISTRAL7B, TINY

own = False

SHAPES = {"tiny": TINY, "7b": LLAMA7B, "7b-gqa": MISTRAL7B, "13b": LLAMA13B}
BLOCK = 16


def _matrix(case):
    """(output rows, input columns, halves) of a case's matrix; the two halves of gate/up feed SwiGLU."""
    sh = SHAPES[case["shape"]]
    hd = sh.head_dim
    return {"qkv": ((sh.n_heads + 2 * sh.n_kv_heads) * hd, sh.d_model, 1), "out": (sh.d_model, sh.n_heads * hd, 1),
            "gate_up": (sh.d_ffn, sh.d_model, 2), "down": (sh.d_model, sh.d_ffn, 1),
            "lm_head": (sh.vocab, sh.d_model, 1)}[case["matrix"]]


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # the smallest product of a decode step: attention output projection of one token; latency counts
        {"name": "linear_7b_out_1", "op": "linear", "shape": "7b", "matrix": "out", "rows": 1, "group": 128,
         "scales": "bf16", "zeros": False},
        # the largest product of a layer for one token, with the norm ahead and the gated activation behind
        {"name": "linear_7b_gate_up_1", "op": "linear", "shape": "7b", "matrix": "gate_up", "rows": 1, "group": 128,
         "scales": "bf16", "zeros": True},
        # q-k-v of a decode batch on the grouped-head shape, fine groups
        {"name": "linear_gqa_qkv_32", "op": "linear", "shape": "7b-gqa", "matrix": "qkv", "rows": 32, "group": 64,
         "scales": "bf16", "zeros": False},
        # down projection of an observation of 256 tokens behind its pending token, scales kept in float32
        {"name": "linear_7b_down_257", "op": "linear", "shape": "7b", "matrix": "down", "rows": 257, "group": 32,
         "scales": "f32", "zeros": False},
        # the largest: gate/up of the mixed step's 1056 rows on the 13B shape
        {"name": "linear_13b_gate_up_1056", "op": "linear", "shape": "13b", "matrix": "gate_up", "rows": 1056,
         "group": 128, "scales": "bf16", "zeros": False},
        # one appended token in each of 32 sequences: one block of each is summarised again
        {"name": "summary_7b_append_32", "op": "summary", "shape": "7b", "seqs": 32, "new_lo": 1, "new_hi": 1,
         "ctx_lo": 512, "ctx_hi": 8192},
        # a long prompt has been prefilled
        {"name": "summary_13b_prompt_16383", "op": "summary", "shape": "13b", "seqs": 1, "new_lo": 16383,
         "new_hi": 16383, "ctx_lo": 16383, "ctx_hi": 16383},
        # one sequence in the middle of a tool-call session
        {"name": "sparse_7b_1", "op": "sparse", "shape": "7b", "rows": 1, "ctx_lo": 1520, "ctx_hi": 1520, "budget": 32,
         "first": 1, "last": 2, "window": 0},
        # one sequence with a very long context on grouped heads
        {"name": "sparse_gqa_long_1", "op": "sparse", "shape": "7b-gqa", "rows": 1, "ctx_lo": 131067, "ctx_hi": 131067,
         "budget": 256, "first": 1, "last": 4, "window": 0},
        # the continuous-batching workload's contexts
        {"name": "sparse_7b_32", "op": "sparse", "shape": "7b", "rows": 32, "ctx_lo": 512, "ctx_hi": 8192, "budget": 64,
         "first": 1, "last": 2, "window": 0},
        # greedy choice inside a grammar for one sequence: only the token is wanted
        {"name": "choose_32000_1", "op": "choose", "vocab": 32000, "rows": 1, "hist_lo": 1520, "hist_hi": 1520,
         "biases": 8, "masks": 1, "sampled": False, "adjusted": False},
        # a sampled batch with long histories whose adjusted logits are wanted too (log-probabilities are reported)
        {"name": "choose_32000_32", "op": "choose", "vocab": 32000, "rows": 32, "hist_lo": 512, "hist_hi": 8192,
         "biases": 64, "masks": 5, "sampled": True, "adjusted": True},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges: rows, contexts and lengths over their logarithm, odd ones among them."""
    op = rng.choice(["linear", "linear", "summary", "sparse", "sparse", "choose"])
    if op == "linear":
        return {"op": op, "shape": rng.choice(["tiny", "7b", "7b-gqa", "13b"]),
                "matrix": rng.choice(["qkv", "out", "gate_up", "down", "lm_head"]), "rows": _log_int(rng, 1, 900),
                "group": rng.choice([32, 64, 128]), "scales": rng.choice(["bf16", "bf16", "f32"]), "zeros": rng.random() < 0.4}
    if op == "choose":
        lo = _log_int(rng, 1, 4096)
        return {"op": op, "vocab": _log_int(rng, 1000, 40000), "rows": _log_int(rng, 1, 32), "hist_lo": lo,
                "hist_hi": rng.randint(lo, 8192), "biases": rng.choice([0, 1, 30, 300]), "masks": rng.choice([0, 1, 7]),
                "sampled": rng.random() < 0.5, "adjusted": rng.random() < 0.5}
    shape = rng.choice(["tiny", "7b", "7b-gqa", "13b"])
    lo = _log_int(rng, 1, 4096)
    if op == "summary":
        seqs = _log_int(rng, 1, 32)
        new = _log_int(rng, 1, min(lo, 16383 // seqs))
        return {"op": op, "shape": shape, "seqs": seqs, "new_lo": rng.randint(1, new), "new_hi": new,
                "ctx_lo": lo, "ctx_hi": rng.randint(lo, 8192)}
    rows = _log_int(rng, 1, 12)
    if rows == 1 and shape == "7b-gqa":
        lo = _log_int(rng, 4096, 131072)
    first, last = rng.randint(0, 2), rng.randint(1, 4)
    return {"op": op, "shape": shape, "rows": rows, "ctx_lo": lo, "ctx_hi": rng.randint(lo, max(lo, 8192)),
            "budget": max(first + last, _log_int(rng, 4, 64 if rows > 1 else 256)), "first": first, "last": last,
            "window": rng.choice([0, 0, SHAPES[shape].window])}


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 29)


def _normal(g, shape, dtype=torch.float32, std=1.0, mean=0.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(mean, std, generator=g)


def _lengths(n, lo, hi, salt=0):
    """Lengths of a case, uniform in [lo, hi]: a function of the case, so that buffers have the same shapes for every seed."""
    return [int(v) for v in np.random.RandomState(((n * 8209 + lo) * 8209 + hi + salt) % (1 << 32)).randint(lo, hi + 1, n)]


def _i32(v):
    return torch.as_tensor(np.ascontiguousarray(v), dtype=torch.int32, device="cuda")


def _el(sh):
    return torch.float32 if sh.dtype == "f32" else torch.bfloat16


def _paged(sh, ctx, rs, g):
    """A layer's pool with the blocks of sequences of these lengths in a seeded order, and the block table."""
    nb = [(c + BLOCK - 1) // BLOCK for c in ctx]
    perm = rs.permutation(sum(nb))
    table = np.full((len(ctx), max(nb)), -1, np.int32)
    at = 0
    for s, n in enumerate(nb):
        table[s, :n] = perm[at:at + n]
        at += n
    pool = _normal(g, (sum(nb), 2, sh.n_kv_heads, BLOCK, sh.head_dim), _el(sh))
    return pool, table


def _prepare_linear(case, seed):
    g = _gen(seed)
    n, k, halves = _matrix(case)
    rows, groups = n * halves, -(-k // case["group"])
    st = {"op": "linear", "n": n, "k": k, "halves": halves, "group": case["group"], "eps": 1e-5,
          # row-major 4-bit codes, two a byte, the even column in the low half; gate rows, then up rows
          "codes": torch.randint(0, 256, (rows, -(-k // 2)), dtype=torch.uint8, device="cuda", generator=g),
          "scales": (0.004 * (0.5 + torch.rand((rows, groups), device="cuda", generator=g))).to(
              torch.bfloat16 if case["scales"] == "bf16" else torch.float32),
          "zeros": torch.randint(5, 12, (rows, groups), dtype=torch.uint8, device="cuda", generator=g) if case["zeros"] else None,
          "x": _normal(g, (case["rows"], k)),
          # q-k-v, gate/up and the LM head follow an RMSNorm
          "gain": _normal(g, (k,), std=0.02, mean=1.0) if case["matrix"] in ("qkv", "gate_up", "lm_head") else None}
    st["x"][:, :: 97] *= 8.0      # a few large columns, as activations have them
    if own:      # the weights, laid out once when a checkpoint is loaded
        import paper_2406_00059_amd as ld
        st["image"] = ld.W4Matrix.pack(st["codes"], st["scales"], st["zeros"], n, k, case["group"], halves)
        st["y"] = torch.empty((case["rows"], n), device="cuda")
        st["scratch"] = torch.empty(max(1, ld.ldk_linear_w4_scratch_bytes(case["rows"], n, k, ld.LDK_SWIGLU if halves == 2 else ld.LDK_STORE)),
                                    dtype=torch.uint8, device="cuda")
    return st


def _prepare_summary(case, seed):
    sh, rs, g = SHAPES[case["shape"]], np.random.RandomState(seed % (1 << 31)), _gen(seed)
    end = _lengths(case["seqs"], case["ctx_lo"], case["ctx_hi"])
    new = [min(e, v) for e, v in zip(end, _lengths(case["seqs"], case["new_lo"], case["new_hi"], 1))]
    pool, table = _paged(sh, end, rs, g)
    ranges = np.stack([np.arange(case["seqs"]), np.array(end) - np.array(new), np.array(end)], 1)
    return {"op": "summary", "hkv": sh.n_kv_heads, "hd": sh.head_dim, "pool": pool, "table": _i32(table), "ranges": _i32(ranges),
            "max_len": max(new),
            "bounds": torch.zeros((pool.shape[0], sh.n_kv_heads, 2, sh.head_dim), dtype=torch.int8, device="cuda"),
            "unit": torch.ones((pool.shape[0], sh.n_kv_heads), device="cuda")}


def _prepare_sparse(case, seed):
    sh, rs, g = SHAPES[case["shape"]], np.random.RandomState(seed % (1 << 31)), _gen(seed)
    ctx = _lengths(case["rows"], case["ctx_lo"], case["ctx_hi"])
    pool, table = _paged(sh, ctx, rs, g)
    keys = pool[:, 0]      # the last block of a sequence may end inside: what its unwritten slots hold is no one's key
    st = {"op": "sparse", "h": sh.n_heads, "hkv": sh.n_kv_heads, "hd": sh.head_dim, "window": case["window"],
          "budget": case["budget"], "first": case["first"], "last": case["last"], "pool": pool, "table": _i32(table),
          "slot": _i32(np.arange(case["rows"])), "ctx": _i32(ctx), "max_ctx": max(ctx),
          "q": _normal(g, (case["rows"], sh.n_heads * sh.head_dim))}
    st["bounds"], st["unit"] = _bounds_of(keys.amin(2).float(), keys.amax(2).float())
    if own:
        import paper_2406_00059_amd as ld
        t = case["rows"]
        st["out"] = torch.empty((t, sh.n_heads, sh.head_dim), device="cuda")
        st["sel"] = torch.empty((t, sh.n_kv_heads, case["budget"]), dtype=torch.int32, device="cuda")
        st["scratch"] = torch.empty(ld.ldk_sparse_attention_scratch_bytes(t, sh.n_heads, sh.n_kv_heads, sh.head_dim, max(ctx), case["window"],
                                                                          case["budget"]), dtype=torch.uint8, device="cuda")
    return st


def _prepare_choose(case, seed):
    rs, g = np.random.RandomState(seed % (1 << 31)), _gen(seed)
    r, v = case["rows"], case["vocab"]
    hist = _lengths(r, case["hist_lo"], case["hist_hi"])
    history = np.full((r, max(hist)), -1, np.int32)
    for i, n in enumerate(hist):      # frequent tokens and rare ones
        history[i, :n] = (v * rs.rand(n) ** 3).astype(np.int32)
    n_bias = [case["biases"]] * r
    words = (v + 31) // 32
    st = {"op": "choose", "v": v, "logits": _normal(g, (r, v), std=3.0), "history": _i32(history), "len": _i32(hist),
          "n_prompt": _i32([n // 2 for n in hist]),
          "penalties": torch.stack([1.0 + 0.3 * torch.rand(r, device="cuda", generator=g), 0.5 * torch.rand(r, device="cuda", generator=g),
                                    0.2 * torch.rand(r, device="cuda", generator=g)], 1).contiguous(),
          "bias_start": _i32(np.concatenate([[0], np.cumsum(n_bias)])) if case["biases"] else None,
          "bias_token": _i32(np.concatenate([rs.permutation(v)[:n] for n in n_bias])) if case["biases"] else None,
          "bias": _normal(g, (sum(n_bias),), std=2.0) if case["biases"] else None,
          "mask": None, "mask_row": None, "temperature": None, "seed": None, "pos": None, "want": case["adjusted"]}
    if case["masks"]:      # grammar states: few tokens allowed in some, nearly all in others; some rows are free
        dense = np.array([0.002, 0.5, 0.05, 0.98, 0.01, 0.3, 0.9])[np.arange(case["masks"]) % 7]
        bits = rs.rand(case["masks"], words * 32) < dense[:, None]
        bits[:, v // 2] = True
        st["mask"] = torch.as_tensor(np.packbits(bits, axis=1, bitorder="little").view(np.int32), device="cuda")
        st["mask_row"] = _i32(np.arange(r) % (case["masks"] + (r > 1)) - (r > 1))
    if case["sampled"]:
        st["temperature"] = torch.as_tensor(np.where(np.arange(r) % 4 == 3, 0.0, 0.4 + 0.8 * rs.rand(r)), dtype=torch.float32, device="cuda")
        st["seed"] = torch.as_tensor(rs.randint(-(1 << 62), 1 << 62, r, dtype=np.int64), device="cuda")
        st["pos"] = st["len"]
    if own:
        import paper_2406_00059_amd as ld
        st["token"] = torch.empty(r, dtype=torch.int32, device="cuda")
        st["adjusted"] = torch.empty((r, v), device="cuda") if case["adjusted"] else None
        st["scratch"] = torch.empty(ld.ldk_choose_scratch_bytes(r, v), dtype=torch.uint8, device="cuda")
    return st


def prepare(case, seed):
    return {"linear": _prepare_linear, "summary": _prepare_summary, "sparse": _prepare_sparse, "choose": _prepare_choose}[case["op"]](case, seed)


# ---------------------------------------------------------------- plain forms

def _plain_linear(s):
    k, grp = s["k"], s["group"]
    c = torch.stack([s["codes"] & 15, s["codes"] >> 4], -1).flatten(1)[:, :k].float()
    z = s["zeros"].float().repeat_interleave(grp, 1)[:, :k] if s["zeros"] is not None else 8.0
    w = (c - z) * s["scales"].float().repeat_interleave(grp, 1)[:, :k]
    x = s["x"]
    if s["gain"] is not None:
        x = x * torch.rsqrt((x * x).mean(1, keepdim=True) + s["eps"]) * s["gain"]
    y = x @ w.t()
    if s["halves"] == 2:
        gate, up = y[:, :s["n"]], y[:, s["n"]:]
        y = gate / (1 + torch.exp(-gate)) * up
    return y


def _unit(top):
    """2^(floor(log2 top) - 6), exact (a quotient that is a power of two): top lies in 64 .. 128 of these units."""
    return torch.where(top > 0, top / torch.frexp(top).mantissa, 2.0) * 2.0 ** -7


def _bounds_of(lo, hi):
    """8-bit bounds [.., 2, hd] (upper, lower) and their unit, a power of two, of keys between lo and hi [.., hd]."""
    top = torch.maximum(lo.abs(), hi.abs()).amax(-1)
    unit = torch.where(top > 0, _unit(top), 1.0)
    up = torch.ceil(hi / unit[..., None]).clamp(max=127)
    down = torch.floor(lo / unit[..., None]).clamp(min=-127)
    return torch.stack([up, down], -2).to(torch.int8).contiguous(), unit.contiguous()


def _plain_summary(s):
    """The bounds of every block that a range's new positions lie in, over the block's positions below the range's end."""
    seq, first, end = s["ranges"].long().unbind(1)
    n = -(-s["max_len"] // BLOCK) + 1
    block = (first // BLOCK)[:, None] + torch.arange(n, device="cuda")      # [ranges, n]
    real = block * BLOCK < end[:, None]
    seq = seq[:, None].expand_as(block)[real]
    end = end[:, None].expand_as(block)[real]
    block = block[real]
    phys = s["table"][seq, block].long()
    keys = s["pool"][phys, 0].float()      # [blocks, Hkv, 16, hd]
    seen = (block[:, None] * BLOCK + torch.arange(BLOCK, device="cuda") < end[:, None])[:, None, :, None]
    inf = float("inf")
    bounds, unit = _bounds_of(keys.masked_fill(~seen, inf).amin(2), keys.masked_fill(~seen, -inf).amax(2))
    s["bounds"][phys], s["unit"][phys] = bounds, unit
    return s["bounds"], s["unit"]


def _plain_sparse(s):
    h, hkv, hd, t, budget = s["h"], s["hkv"], s["hd"], s["q"].shape[0], s["budget"]
    dev, inf = "cuda", float("inf")
    q = s["q"].view(t, hkv, h // hkv, hd)
    ctx = s["ctx"].long()
    start = (ctx - s["window"]).clamp(min=0) if s["window"] else torch.zeros_like(ctx)
    nb = -(-s["max_ctx"] // BLOCK)
    block = torch.arange(nb, device=dev)
    b0, b1 = start // BLOCK, -(-ctx // BLOCK)
    live = (block >= b0[:, None]) & (block < b1[:, None])
    kept = live & ((block < b0[:, None] + s["first"]) | (block >= b1[:, None] - s["last"]))
    phys = s["table"][s["slot"].long()][:, :nb].long().clamp(min=0)
    # scores: integers (below 2^24, so that float32 sums are exact) times powers of two
    v = _unit(q.abs().amax(-1))
    qi = torch.round(q / v[..., None]).clamp(-127, 127)
    bounds = s["bounds"][phys].permute(0, 2, 1, 3, 4).float()      # [t, hkv, nb, 2, hd]
    both = torch.cat([qi.clamp(min=0), qi.clamp(max=0)], -1).transpose(-1, -2).contiguous()      # [t, hkv, 2 hd, g]
    dots = bounds.flatten(3) @ both
    score = (dots * v[:, :, None, :] * s["unit"][phys].transpose(1, 2)[..., None]).amax(-1)
    score = torch.where(kept[:, None], inf, torch.where(live[:, None], score, -inf))
    n = min(budget, nb)
    sel = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :n]
    sel = torch.where(torch.arange(n, device=dev) < live.sum(1)[:, None, None], sel, nb)      # fewer blocks than the budget
    sel = torch.sort(sel, -1).values
    got = sel < nb
    at = torch.gather(phys[:, None].expand(t, hkv, nb), 2, sel.clamp(max=nb - 1))
    head = torch.arange(hkv, device=dev)[None, :, None]
    keys = s["pool"][at, 0, head].float()      # [t, hkv, n, 16, hd]
    vals = s["pool"].view(-1, 2, hkv, hd, BLOCK)[at, 1, head].float()      # values lie transposed in a block
    pos = sel[..., None] * BLOCK + torch.arange(BLOCK, device=dev)
    seen = got[..., None] & (pos >= start[:, None, None, None]) & (pos < ctx[:, None, None, None])
    sc = (keys.flatten(2, 3) @ q.transpose(-1, -2).contiguous()) / math.sqrt(hd)      # [t, hkv, n 16, g]
    sc = sc.masked_fill(~seen.flatten(2)[..., None], -inf)
    top = sc.amax(2, keepdim=True)
    p = torch.exp(sc - torch.where(top > -inf, top, 0.0))
    total = p.sum(2)      # [t, hkv, g]
    p = p.view(t, hkv, n, BLOCK, -1)
    # sum over the positions of a block, then over blocks: one product with the dimensions of a value in rows
    vv = vals.permute(0, 1, 3, 2, 4).reshape(t, hkv, hd, n * BLOCK)
    out = (vv @ p.flatten(2, 3)).transpose(-1, -2) / torch.where(total > 0, total, 1.0)[..., None]
    full = torch.full((t, hkv, budget), -1, dtype=torch.int32, device=dev)
    full[..., :n] = torch.where(got, sel, -1)
    return out.reshape(t, h, hd), full


def _gumbel(seed, pos, v):
    """-log(-log u) [rows, v], u from the SplitMix64 output function at counter pos v + i + 1."""
    def shr(z, n):
        return (z >> n) & ((1 << (64 - n)) - 1)
    z = seed[:, None] + (pos.long()[:, None] * v + torch.arange(v, device=seed.device) + 1) * (0x9E3779B97F4A7C15 - (1 << 64))
    z = (z ^ shr(z, 30)) * (0xBF58476D1CE4E5B9 - (1 << 64))
    z = (z ^ shr(z, 27)) * (0x94D049BB133111EB - (1 << 64))
    z = z ^ shr(z, 31)
    u = (shr(z, 41).float() + 0.5) * 2.0 ** -23
    return -torch.log(-torch.log(u))


def _plain_choose(s):
    v, l = s["v"], s["logits"]
    r, n = l.shape[0], s["history"].shape[1]
    at = torch.arange(n, device="cuda")
    real = at < s["len"][:, None]
    answer = real & (at >= s["n_prompt"][:, None])
    tok = s["history"].long().clamp(min=0)
    seen = torch.zeros((r, v), dtype=torch.int32, device="cuda").scatter_add_(1, tok, real.int()) > 0
    count = torch.zeros((r, v), dtype=torch.int32, device="cuda").scatter_add_(1, tok, answer.int())
    rep, pres, freq = s["penalties"][:, :, None].unbind(1)
    l = torch.where(seen, torch.where(l > 0, l / rep, l * rep), l)
    l = l - (freq * count + pres * (count > 0))
    if s["bias"] is not None:      # the same number of entries for every row here, all tokens of a row distinct
        l = l.scatter_add(1, s["bias_token"].long().view(r, -1), s["bias"].view(r, -1))
    if s["mask"] is not None:
        ids = torch.arange(v, device="cuda")
        allowed = (s["mask"][:, ids // 32] >> (ids % 32)) & 1
        l = torch.where((s["mask_row"][:, None] < 0) | (allowed[s["mask_row"].clamp(min=0).long()] > 0), l, float("-inf"))
    score = l
    if s["temperature"] is not None:
        temp = s["temperature"][:, None]
        drawn = l * torch.where(temp > 0, 1 / temp, 1.0) + _gumbel(s["seed"], s["pos"], v)
        score = torch.where(temp > 0, drawn, l)
    best = score.amax(1, keepdim=True)
    first = torch.where(score == best, torch.arange(v, device="cuda"), v).amin(1)
    token = torch.where(best[:, 0] > float("-inf"), first, -1).int()
    return (token, l) if s["want"] else (token,)


# ---------------------------------------------------------------- one pass

def run(s):
    if not own:
        return {"linear": _plain_linear, "summary": _plain_summary, "sparse": _plain_sparse, "choose": _plain_choose}[s["op"]](s)
    import paper_2406_00059_amd as ld
    if s["op"] == "linear":
        ld.ldk_linear_w4(s["image"], s["x"], s["y"], ld.LDK_SWIGLU if s["halves"] == 2 else ld.LDK_STORE, g=s["gain"], eps=s["eps"],
                         scratch=s["scratch"])
        return s["y"]
    if s["op"] == "summary":
        ld.ldk_kv_summary(s["pool"], s["table"], s["ranges"], s["max_len"], s["hkv"], s["hd"], s["bounds"], s["unit"])
        return s["bounds"], s["unit"]
    if s["op"] == "sparse":
        ld.ldk_sparse_attention(s["q"], s["h"] * s["hd"], s["pool"], s["bounds"], s["unit"], s["table"], s["slot"], s["ctx"], s["max_ctx"],
                                s["h"], s["hkv"], s["hd"], s["budget"], s["first"], s["last"], s["out"], s["sel"], s["scratch"],
                                window=s["window"])
        return s["out"], s["sel"]
    ld.ldk_choose(s["logits"], s["token"], history=s["history"], history_len=s["len"], n_prompt=s["n_prompt"], penalties=s["penalties"],
                  bias_start=s["bias_start"], bias_token=s["bias_token"], bias=s["bias"], mask=s["mask"], mask_row=s["mask_row"],
                  temperature=s["temperature"], seed=s["seed"], pos=s["pos"], adjusted=s["adjusted"], scratch=s["scratch"])
    return (s["token"], s["adjusted"]) if s["want"] else (s["token"],)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["op"] == "linear":
        n, k, halves = _matrix(case)
        rows, groups, t = n * halves, -(-k // case["group"]), case["rows"]
        per = (2 if case["scales"] == "bf16" else 4) + (1 if case["zeros"] else 0)
        return {"bytes": rows * -(-k // 2) + rows * groups * per + 4 * t * (k + n), "flops": 2 * t * rows * k}
    if case["op"] == "choose":
        r, v = case["rows"], case["vocab"]
        hist = sum(_lengths(r, case["hist_lo"], case["hist_hi"]))
        return {"bytes": 4 * r * v * (2 if case["adjusted"] else 1) + 4 * hist + case["masks"] * v // 8 + 8 * r * case["biases"] + 4 * r,
                "flops": r * v * 4}
    sh = SHAPES[case["shape"]]
    el = 4 if sh.dtype == "f32" else 2
    hkv, hd = sh.n_kv_heads, sh.head_dim
    if case["op"] == "summary":
        end = _lengths(case["seqs"], case["ctx_lo"], case["ctx_hi"])
        new = [min(e, v) for e, v in zip(end, _lengths(case["seqs"], case["new_lo"], case["new_hi"], 1))]
        pos = sum(e - (e - n) // BLOCK * BLOCK for e, n in zip(end, new))
        blocks = sum(-(-e // BLOCK) - (e - n) // BLOCK for e, n in zip(end, new))
        return {"bytes": pos * hkv * hd * el + blocks * hkv * (2 * hd + 4), "flops": 2 * pos * hkv * hd}
    nbytes, flops, w = 0, 0, case["window"]
    for c in _lengths(case["rows"], case["ctx_lo"], case["ctx_hi"]):
        seen = -(-c // BLOCK) - (max(0, c - w) // BLOCK if w else 0)
        taken = min(seen, case["budget"])
        nbytes += hkv * (seen * (2 * hd + 4) + taken * 2 * BLOCK * hd * el + case["budget"] * 4) + 8 * sh.n_heads * hd
        flops += sh.n_heads * (seen * 4 * hd + taken * BLOCK * 4 * hd)
    return {"bytes": nbytes, "flops": flops}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_linear(s):
    w = torch.empty((s["codes"].shape[0], s["codes"].shape[1] * 2), dtype=torch.float64, device="cuda")
    w[:, 0::2] = s["codes"] % 16
    w[:, 1::2] = torch.div(s["codes"], 16, rounding_mode="floor")
    w = w[:, :s["k"]].contiguous()
    for j in range(s["scales"].shape[1]):
        cols = slice(j * s["group"], min(s["k"], (j + 1) * s["group"]))
        w[:, cols] -= 8 if s["zeros"] is None else s["zeros"][:, j:j + 1].double()
        w[:, cols] *= s["scales"][:, j:j + 1].double()
    x = s["x"].double()
    if s["gain"] is not None:
        x = x / (x.pow(2).sum(1, keepdim=True) / s["k"] + s["eps"]).sqrt() * s["gain"].double()
    y = torch.mm(x, w.t().contiguous())
    return torch.sigmoid(y[:, :s["n"]]) * y[:, :s["n"]] * y[:, s["n"]:] if s["halves"] == 2 else y


def _exact_sparse(s):
    """Row by row and head by head on the host; the choice of blocks in integers."""
    h, hkv, hd, w = s["h"], s["hkv"], s["hd"], s["window"]
    g = h // hkv
    q = s["q"].double().cpu().numpy().reshape(-1, h, hd)
    ctx, table, slot = s["ctx"].tolist(), s["table"].cpu().numpy(), s["slot"].tolist()
    out = np.zeros_like(q)
    for t in range(q.shape[0]):
        start = max(0, ctx[t] - w) if w else 0
        lo, hi = start // BLOCK, -(-ctx[t] // BLOCK)
        if hi <= lo:
            continue
        phys = torch.as_tensor(table[slot[t], lo:hi], device="cuda").long()
        bounds, unit = s["bounds"][phys].cpu().numpy().astype(np.int64), s["unit"][phys].double().cpu().numpy()
        for j in range(hkv):
            score = np.full(hi - lo, -np.inf)
            for i in range(j * g, j * g + g):
                top = np.abs(q[t, i]).max()
                step = 2.0 ** (math.floor(math.log2(top)) - 6) if top > 0 else 2.0 ** -6
                qi = np.clip(np.rint(q[t, i] / step), -127, 127).astype(np.int64)
                dot = bounds[:, j, 0] @ np.maximum(qi, 0) + bounds[:, j, 1] @ np.minimum(qi, 0)
                score = np.maximum(score, dot * step * unit[:, j])
            score[:s["first"]] = np.inf
            score[max(0, hi - lo - s["last"]):] = np.inf
            took = np.sort(np.argsort(-score, kind="stable")[:s["budget"]])
            blocks = s["pool"][phys[torch.as_tensor(took, device="cuda")]][:, :, j].double().cpu().numpy()
            keys = blocks[:, 0].reshape(-1, hd)
            vals = blocks[:, 1].reshape(len(took), hd, BLOCK).transpose(0, 2, 1).reshape(-1, hd)
            pos = ((took + lo)[:, None] * BLOCK + np.arange(BLOCK)).reshape(-1)
            ok = (pos >= start) & (pos < ctx[t])
            sc = keys[ok] @ q[t, j * g:j * g + g].T / math.sqrt(hd)
            p = np.exp(sc - sc.max(0))
            out[t, j * g:j * g + g] = (p / p.sum(0)).T @ vals[ok]
    return torch.from_numpy(out)


def _exact_choose(s):
    """The adjusted logits, one row after another."""
    l = s["logits"].double().cpu().numpy()
    hist, n, start = s["history"].cpu().numpy(), s["len"].tolist(), s["n_prompt"].tolist()
    pen = s["penalties"].double().cpu().numpy()
    v = s["v"]
    for r in range(l.shape[0]):
        seen = np.bincount(hist[r, :n[r]], minlength=v) > 0
        count = np.bincount(hist[r, start[r]:n[r]], minlength=v)
        rep, pres, freq = pen[r]
        l[r] = np.where(seen, np.where(l[r] > 0, l[r] / rep, l[r] * rep), l[r]) - freq * count - pres * (count > 0)
        if s["bias"] is not None:
            a, b = s["bias_start"][r].item(), s["bias_start"][r + 1].item()
            l[r, s["bias_token"][a:b].cpu().numpy()] += s["bias"][a:b].double().cpu().numpy()
        m = -1 if s["mask"] is None else s["mask_row"][r].item()
        if m >= 0:
            bits = np.unpackbits(s["mask"][m].cpu().numpy().view(np.uint8), bitorder="little")[:v]
            l[r, bits == 0] = -np.inf
    return torch.from_numpy(l)


def exact(case, seed):
    """What run() returns, from the definitions in 64 bits; None in the place of whole numbers."""
    s = prepare(case, seed)
    if case["op"] == "linear":
        return _exact_linear(s)
    if case["op"] == "summary":
        unit = s["unit"].double().cpu().numpy()
        table = s["table"].cpu().numpy()
        for seq, first, end in s["ranges"].tolist():
            for b in range(first // BLOCK, -(-end // BLOCK)):
                k = s["pool"][int(table[seq, b]), 0, :, :end - b * BLOCK].double().abs().amax((1, 2)).cpu().numpy()
                unit[table[seq, b]] = [2.0 ** (math.floor(math.log2(x)) - 6) if x > 0 else 1.0 for x in k]
        return None, torch.from_numpy(unit)
    if case["op"] == "sparse":
        return _exact_sparse(s), None
    return (None, _exact_choose(s)) if s["want"] else None
