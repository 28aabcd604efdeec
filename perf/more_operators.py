"""The operators of an 8-bit paged cache, as cases to time and to compare.

Four operators, each in its plain form (elementary torch operations) and through the package's entry points:

  write    norms of a row's q and k heads, the position rotation (both pair layouts, whole heads or a part, frequencies scaled for
           long contexts) and the append of keys and values in 8 bits; then what was stored is read back into a cache of the model's type.
  move     cached positions of whole sequences into an 8-bit cache and back: a sequence that waits for a tool is set aside at half its size.
  decode   attention of one new token a row over the 8-bit cache.
  prefill  attention of prompt and observation rows over the 8-bit cache.

An 8-bit vector of one position and KV head is 127 >= |c| times 2^e: e = floor(log2 max |x|) - 6 (at least -126), c = x 2^-e rounded to
nearest, ties to even.  Scores may be capped (cap tanh(s / cap)) and may get a bias slope (j - p); rows may be kept from positions ahead
of their document's start or outside a band, and rows of a prefix see all of it.

Shapes are the repository's own decoder shapes; batch sizes, contexts and chunk lengths are those of its workloads (one sequence at a
context of some 1500 tokens, 32 sequences U[512, 8192], observations of 256 tokens behind their pending token, the mixed step of 1056
rows).  Block tables are seeded permutations of the pool.
"""
import math

import numpy as np
import torch

from workloads import LLAMA7B, LLAMA13B, MISTRAL7B, TINY

own = False

SHAPES = {"tiny": TINY, "7b": LLAMA7B, "7b-gqa": MISTRAL7B, "13b": LLAMA13B}
BLOCK = 16
EPS = 1e-5


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # one token of one sequence in the middle of a tool-call session; latency counts
        {"name": "write_7b_1", "op": "write", "shape": "7b", "chunks": 0, "chunk": 0, "singles": 1, "ctx_lo": 1519, "ctx_hi": 1519,
         "rot": 128, "interleaved": False, "norm": False, "factor": 1.0},
        # a decode batch of a model with head norms, half of each head rotated in neighbouring pairs, context stretched eightfold: the
        # first layer of a step, where the angles are made
        {"name": "write_gqa_32", "op": "write", "shape": "7b-gqa", "chunks": 0, "chunk": 0, "singles": 32, "ctx_lo": 512, "ctx_hi": 65536,
         "rot": 64, "interleaved": True, "norm": True, "factor": 8.0},
        # the mixed step's rows on the 13B shape: four observations with their pending tokens beside 28 decoding sequences
        {"name": "write_13b_1056", "op": "write", "shape": "13b", "chunks": 4, "chunk": 257, "singles": 28, "ctx_lo": 512, "ctx_hi": 8192,
         "rot": 128, "interleaved": False, "norm": False, "factor": 1.0},
        # a sequence waits for its tool
        {"name": "move_gqa_1", "op": "move", "shape": "7b-gqa", "seqs": 1, "len_lo": 1520, "len_hi": 1520},
        # eight long ones do
        {"name": "move_13b_8", "op": "move", "shape": "13b", "seqs": 8, "len_lo": 512, "len_hi": 8192},
        # one sequence in the middle of a tool-call session
        {"name": "decode_7b_1", "op": "decode", "shape": "7b", "rows": 1, "pad": 0, "ctx_lo": 1520, "ctx_hi": 1520, "window": 0, "cap": 0.0,
         "bias": False, "doc": False},
        # one sequence with a very long context on grouped heads
        {"name": "decode_gqa_long_1", "op": "decode", "shape": "7b-gqa", "rows": 1, "pad": 0, "ctx_lo": 131067, "ctx_hi": 131067, "window": 0,
         "cap": 0.0, "bias": False, "doc": False},
        # the continuous-batching workload's contexts
        {"name": "decode_7b_32", "op": "decode", "shape": "7b", "rows": 32, "pad": 0, "ctx_lo": 512, "ctx_hi": 8192, "window": 0, "cap": 0.0,
         "bias": False, "doc": False},
        # a small batch in a graph of eight rows, one of them without a sequence: capped scores, distance bias, packed documents
        {"name": "decode_13b_capped_8", "op": "decode", "shape": "13b", "rows": 8, "pad": 1, "ctx_lo": 1, "ctx_hi": 2048, "window": 0,
         "cap": 30.0, "bias": True, "doc": True},
        # an observation of 256 tokens behind its pending token
        {"name": "prefill_7b_257", "op": "prefill", "shape": "7b", "seqs": 1, "rows_lo": 257, "rows_hi": 257, "before_lo": 1263,
         "before_hi": 1263, "window": 0, "cap": 0.0, "bias": False, "prefix": False, "doc": False},
        # the largest: a long prompt on grouped heads with the shape's band
        {"name": "prefill_gqa_prompt_8191", "op": "prefill", "shape": "7b-gqa", "seqs": 1, "rows_lo": 8191, "rows_hi": 8191, "before_lo": 0,
         "before_hi": 0, "window": 4096, "cap": 0.0, "bias": False, "prefix": False, "doc": False},
        # observations of a mixed step: capped scores, half of each chunk a prefix that sees all of itself, packed documents
        {"name": "prefill_13b_capped_4", "op": "prefill", "shape": "13b", "seqs": 4, "rows_lo": 65, "rows_hi": 257, "before_lo": 512,
         "before_hi": 4096, "window": 0, "cap": 50.0, "bias": False, "prefix": True, "doc": True},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges: rows, contexts and lengths over their logarithm, odd ones among them."""
    op = rng.choice(["write", "write", "move", "decode", "decode", "decode", "prefill", "prefill", "prefill"])
    shape = rng.choice(["tiny", "7b", "7b-gqa", "13b"])
    sh = SHAPES[shape]
    if op == "write":
        chunks = rng.choice([0, 0, 1, 3])
        chunk = _log_int(rng, 2, 257) if chunks else 0
        lo = _log_int(rng, 1, 8192)
        return {"op": op, "shape": shape, "chunks": chunks, "chunk": chunk, "singles": _log_int(rng, 1, 64), "ctx_lo": lo,
                "ctx_hi": rng.randint(lo, 65536), "rot": rng.choice([sh.head_dim, sh.head_dim, sh.head_dim // 2, 2 * rng.randint(1, sh.head_dim // 2)]),
                "interleaved": rng.random() < 0.5, "norm": rng.random() < 0.5, "factor": rng.choice([1.0, 1.0, 4.0, 32.0])}
    if op == "move":
        lo = _log_int(rng, 1, 4096)
        return {"op": op, "shape": shape, "seqs": _log_int(rng, 1, 8), "len_lo": lo, "len_hi": rng.randint(lo, 8192)}
    window = rng.choice([0, 0, sh.window, _log_int(rng, 1, 4096)])
    if op == "decode":
        rows = _log_int(rng, 1, 32)
        lo = _log_int(rng, 1, 4096)
        if rows == 1 and shape == "7b-gqa":
            lo = _log_int(rng, 4096, 131072)
        return {"op": op, "shape": shape, "rows": rows, "pad": rng.choice([0, 0, 1]) if rows > 1 else 0, "ctx_lo": lo,
                "ctx_hi": rng.randint(lo, max(lo, 8192)), "window": window, "cap": rng.choice([0.0, 0.0, 15.0, 50.0]), "bias": rng.random() < 0.3,
                "doc": rng.random() < 0.3}
    seqs = rng.choice([1, 1, 2, 5])
    rows = _log_int(rng, 1, 2500 // seqs ** 2)
    before = _log_int(rng, 1, 4096)
    return {"op": op, "shape": shape, "seqs": seqs, "rows_lo": rng.randint(1, rows), "rows_hi": rows, "before_lo": rng.choice([0, before]),
            "before_hi": before, "window": window, "cap": rng.choice([0.0, 0.0, 15.0, 50.0]), "bias": rng.random() < 0.3,
            "prefix": rng.random() < 0.3, "doc": rng.random() < 0.3}


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 31)


def _normal(g, shape, std=1.0, mean=0.0):
    return torch.empty(shape, device="cuda").normal_(mean, std, generator=g)


def _lengths(n, lo, hi, salt=0):
    """Lengths of a case, uniform in [lo, hi]: a function of the case, so that buffers have the same shapes for every seed."""
    return [int(v) for v in np.random.RandomState(((n * 8209 + lo) * 8209 + hi + salt) % (1 << 32)).randint(lo, hi + 1, n)]


def _i32(v):
    return torch.as_tensor(np.ascontiguousarray(v), dtype=torch.int32, device="cuda")


def _el(sh):
    return torch.float32 if sh.dtype == "f32" else torch.bfloat16


def _tables(blocks, rs):
    """A block table whose sequences hold the given logical blocks, in a seeded order of the pool; the number of blocks."""
    total = sum(len(b) for b in blocks)
    perm, at = rs.permutation(total), 0
    table = np.full((len(blocks), max(max(b, default=0) for b in blocks) + 1), -1, np.int32)
    for s, b in enumerate(blocks):
        table[s, list(b)] = perm[at:at + len(b)]
        at += len(b)
    return table, total


def _cache(sh, lengths, rs, g):
    """An 8-bit layer of sequences of these lengths: keys and values as their projections have them, some dimensions larger than others."""
    table, n = _tables([range(-(-v // BLOCK)) for v in lengths], rs)
    codes = torch.empty((n, 2, sh.n_kv_heads, BLOCK, sh.head_dim), dtype=torch.int8, device="cuda")
    expo = torch.empty((n, 2, sh.n_kv_heads, BLOCK), dtype=torch.int8, device="cuda")
    for a in range(0, n, 1024):
        b = min(n, a + 1024)
        x = _normal(g, (b - a, 2, sh.n_kv_heads, BLOCK, sh.head_dim))
        x[:, 0, :, :, 5::32] *= 4.0
        e = torch.frexp(x.abs().amax(-1)).exponent - 7
        c = torch.round(x * ((e + 127) << 23).view(torch.float32)[..., None].reciprocal()).clamp(-127, 127).to(torch.int8)
        codes[a:b, 0] = c[:, 0]
        codes[a:b, 1] = c[:, 1].transpose(-1, -2).reshape(c[:, 1].shape)      # values lie transposed in a block
        expo[a:b] = e
    return table, codes, expo


def _prepare_write(case, seed):
    sh, rs, g = SHAPES[case["shape"]], np.random.RandomState(seed % (1 << 31)), _gen(seed)
    h, hkv, hd = sh.n_heads, sh.n_kv_heads, sh.head_dim
    count = [case["chunk"]] * case["chunks"] + [1] * case["singles"]
    first = _lengths(len(count), case["ctx_lo"], case["ctx_hi"])
    t = sum(count)
    table, n = _tables([range(f // BLOCK, -(-(f + c) // BLOCK)) for f, c in zip(first, count)], rs)
    qkv = _normal(g, (t, (h + 2 * hkv) * hd))
    qkv[:, 3::64] *= 6.0      # some dimensions are larger than others
    pos = np.concatenate([np.arange(f, f + c) for f, c in zip(first, count)])
    stretched = case["factor"] != 1.0
    st = {"op": "write", "h": h, "hkv": hkv, "hd": hd, "rot": case["rot"], "interleaved": case["interleaved"], "base": sh.rope_base,
          # wavelengths longer than the original context are stretched whole, those a quarter as long not at all
          "scaling": {"factor": case["factor"], "low": 1.0, "high": 4.0, "original": 8192, "attention": 1.1} if stretched else None,
          "qkv": qkv, "pos": _i32(pos), "slot": _i32(np.repeat(np.arange(len(count)), count)), "table": _i32(table),
          "ranges": _i32(np.stack([np.arange(len(count)), first, np.add(first, count)], 1)), "max_len": max(count),
          "q_gain": _normal(g, (hd,), 0.1, 1.0) if case["norm"] else None, "k_gain": _normal(g, (hd,), 0.1, 1.0) if case["norm"] else None,
          "codes": torch.zeros((n, 2, hkv, BLOCK, hd), dtype=torch.int8, device="cuda"),
          "expo": torch.zeros((n, 2, hkv, BLOCK), dtype=torch.int8, device="cuda"),
          "pool": torch.zeros((n, 2, hkv, BLOCK, hd), dtype=_el(sh), device="cuda"),
          "q": torch.empty((t, h * hd), device="cuda"), "cos_sin": torch.empty((t, case["rot"] // 2, 2), device="cuda")}
    if not stretched:      # a later layer: the step's angles are there
        angle = st["pos"].double()[:, None] * torch.pow(float(sh.rope_base), -2.0 * torch.arange(case["rot"] // 2, device="cuda", dtype=torch.float64) / case["rot"])
        st["cos_sin"].copy_(torch.stack([torch.cos(angle), torch.sin(angle)], -1))
    return st


def _prepare_move(case, seed):
    sh, rs, g = SHAPES[case["shape"]], np.random.RandomState(seed % (1 << 31)), _gen(seed)
    length = _lengths(case["seqs"], case["len_lo"], case["len_hi"])
    blocks = [range(-(-v // BLOCK)) for v in length]
    table, n = _tables(blocks, rs)
    shape = (n, 2, sh.n_kv_heads, BLOCK, sh.head_dim)
    return {"op": "move", "hkv": sh.n_kv_heads, "hd": sh.head_dim, "pool": _normal(g, shape).to(_el(sh)), "table": _i32(table),
            "table8": _i32(_tables(blocks, rs)[0]), "back": _i32(_tables(blocks, rs)[0]), "restored": torch.zeros(shape, dtype=_el(sh), device="cuda"),
            "ranges": _i32(np.stack([np.arange(case["seqs"]), np.zeros(case["seqs"], int), length], 1)), "max_len": max(length),
            "codes": torch.zeros(shape, dtype=torch.int8, device="cuda"), "expo": torch.zeros(shape[:4], dtype=torch.int8, device="cuda")}


def _slopes(h):
    return torch.as_tensor(2.0 ** (-8.0 * (np.arange(h) + 1) / h), dtype=torch.float32, device="cuda")


def _contexts(case):
    ctx = _lengths(case["rows"], case["ctx_lo"], case["ctx_hi"])
    return [0 if i >= case["rows"] - case["pad"] else c for i, c in enumerate(ctx)]


def _starts(case, lengths):
    """First position of each row's document."""
    return [v // 3 if case["doc"] and i % 2 == 0 else 0 for i, v in enumerate(lengths)]


def _prepare_decode(case, seed):
    sh, rs, g = SHAPES[case["shape"]], np.random.RandomState(seed % (1 << 31)), _gen(seed)
    ctx = _contexts(case)
    table, codes, expo = _cache(sh, ctx, rs, g)
    t = len(ctx)
    st = {"op": "decode", "h": sh.n_heads, "hkv": sh.n_kv_heads, "hd": sh.head_dim, "window": case["window"], "cap": case["cap"],
          "slopes": _slopes(sh.n_heads) if case["bias"] else None, "codes": codes, "expo": expo, "table": _i32(table), "slot": _i32(np.arange(t)),
          "ctx": _i32(ctx), "max_ctx": max(ctx), "first": _i32(_starts(case, ctx)) if case["doc"] else None,
          "q": _normal(g, (t, sh.n_heads * sh.head_dim))}
    if own:
        import paper_2406_00059_amd as ld
        st["out"] = torch.empty((t, sh.n_heads, sh.head_dim), device="cuda")
        st["scratch"] = torch.empty(ld.ldk_attention_q8_scratch_bytes(t, sh.n_heads, sh.n_kv_heads, sh.head_dim, max(ctx), case["window"]),
                                    dtype=torch.uint8, device="cuda")
    return st


def _segments(case):
    """(rows, positions before them, first position of the document, prefix) of each sequence."""
    n = _lengths(case["seqs"], case["rows_lo"], case["rows_hi"])
    before = _lengths(case["seqs"], case["before_lo"], case["before_hi"], 1)
    prefix = [b + (v + 1) // 2 if case["prefix"] else 0 for b, v in zip(before, n)]
    return n, before, _starts(case, before), prefix


def _prepare_prefill(case, seed):
    sh, rs, g = SHAPES[case["shape"]], np.random.RandomState(seed % (1 << 31)), _gen(seed)
    n, before, first, prefix = _segments(case)
    table, codes, expo = _cache(sh, [b + v for b, v in zip(before, n)], rs, g)
    t, start = sum(n), np.concatenate([[0], np.cumsum(n)])
    # tiles of up to 128 rows of a sequence: (first row, rows, position of the first row, table row, first visible position, prefix)
    tiles = [(start[s] + i, min(128, n[s] - i), before[s] + i, s, first[s], prefix[s]) for s in range(len(n)) for i in range(0, n[s], 128)]
    st = {"op": "prefill", "h": sh.n_heads, "hkv": sh.n_kv_heads, "hd": sh.head_dim, "window": case["window"], "cap": case["cap"],
          "slopes": _slopes(sh.n_heads) if case["bias"] else None, "codes": codes, "expo": expo, "table": _i32(table), "tiles": _i32(np.array(tiles)),
          "seqs": (n, before, first, prefix), "max_pos": max(b + v for b, v in zip(before, n)) - 1,
          "q": _normal(g, (t, sh.n_heads * sh.head_dim))}
    if own:
        import paper_2406_00059_amd as ld
        st["out"] = torch.empty((t, sh.n_heads, sh.head_dim), device="cuda")
        st["scratch"] = torch.empty(ld.ldk_prefill_attention_q8_scratch_bytes(len(tiles), sh.n_heads, sh.n_kv_heads, sh.head_dim, st["max_pos"],
                                                                              case["window"]), dtype=torch.uint8, device="cuda")
    return st


def prepare(case, seed):
    return {"write": _prepare_write, "move": _prepare_move, "decode": _prepare_decode, "prefill": _prepare_prefill}[case["op"]](case, seed)


# ---------------------------------------------------------------- plain forms

def _power(e):
    """2^e in float64, e of a whole type."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _quantise(x):
    """Codes and exponents of float64 vectors [.., hd]."""
    top = x.abs().amax(-1)
    e = torch.where(top > 0, torch.frexp(top).exponent.long() - 7, -126).clamp(min=-126)
    return torch.round(x * _power(-e)[..., None]).clamp(-127, 127).to(torch.int8), e.to(torch.int8)


def _places(table, ranges, max_len):
    """Sequence and position of every position of the ranges."""
    at = ranges[:, 1].long()[:, None] + torch.arange(max_len, device="cuda")
    real = at < ranges[:, 2].long()[:, None]
    return ranges[:, 0].long()[:, None].expand_as(at)[real], at[real]


def _store(codes, expo, phys, slot, k, v):
    """Keys and values [n, Hkv, hd] in 8 bits into blocks phys, slots slot."""
    n, hkv, hd = k.shape
    (ck, ek), (cv, ev) = _quantise(k), _quantise(v)
    codes[phys, 0, :, slot] = ck
    codes.view(-1, 2, hkv, hd, BLOCK)[phys, 1, :, :, slot] = cv
    expo[phys, 0, :, slot] = ek
    expo[phys, 1, :, slot] = ev


def _read_back(codes, expo, table, pool, back, ranges, max_len):
    seq, at = _places(table, ranges, max_len)
    phys, to, slot = table[seq, at // BLOCK].long(), back[seq, at // BLOCK].long(), at % BLOCK
    n, _, hkv, _, hd = codes.shape
    unit = _power(expo[phys, :, :, slot]).float()      # [n, 2, hkv]
    pool[to, 0, :, slot] = (codes[phys, 0, :, slot] * unit[:, 0, :, None]).to(pool.dtype)
    pool.view(-1, 2, hkv, hd, BLOCK)[to, 1, :, :, slot] = (codes.view(-1, 2, hkv, hd, BLOCK)[phys, 1, :, :, slot] * unit[:, 1, :, None]).to(pool.dtype)


def _plain_write(s):
    h, hkv, hd, rot = s["h"], s["hkv"], s["hd"], s["rot"]
    t = s["qkv"].shape[0]
    if s["scaling"]:
        c = s["scaling"]
        f = torch.pow(float(s["base"]), -2.0 * torch.arange(rot // 2, device="cuda", dtype=torch.float64) / rot)
        g = ((c["original"] * f / (2 * math.pi) - c["low"]) / (c["high"] - c["low"])).clamp(0, 1)
        angle = s["pos"].double()[:, None] * (f * ((1 - g) / c["factor"] + g))
        s["cos_sin"].copy_(float(np.float32(c["attention"])) * torch.stack([torch.cos(angle), torch.sin(angle)], -1))
    x = s["qkv"].double().view(t, h + 2 * hkv, hd)
    q, k, v = x[:, :h], x[:, h:h + hkv], x[:, h + hkv:]
    if s["q_gain"] is not None:
        q = q / torch.sqrt((q * q).mean(-1, keepdim=True) + float(np.float32(EPS))) * s["q_gain"].double()
        k = k / torch.sqrt((k * k).mean(-1, keepdim=True) + float(np.float32(EPS))) * s["k_gain"].double()
    x = torch.cat([q, k], 1)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if s["interleaved"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    cos, sin = s["cos_sin"].double()[:, None, :, 0], s["cos_sin"].double()[:, None, :, 1]
    a, b = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([a, b], -1).flatten(-2) if s["interleaved"] else torch.cat([a, b], -1)
    x = torch.cat([turned, x[..., rot:]], -1)
    s["q"].copy_(x[:, :h].reshape(t, h * hd))
    phys = s["table"][s["slot"].long(), s["pos"].long() // BLOCK].long()
    _store(s["codes"], s["expo"], phys, s["pos"].long() % BLOCK, x[:, h:], v)
    _read_back(s["codes"], s["expo"], s["table"], s["pool"], s["table"], s["ranges"], s["max_len"])
    return s["q"], s["pool"]


def _plain_move(s):
    hkv, hd = s["hkv"], s["hd"]
    seq, at = _places(s["table"], s["ranges"], s["max_len"])
    phys, to, slot = s["table"][seq, at // BLOCK].long(), s["table8"][seq, at // BLOCK].long(), at % BLOCK
    k = s["pool"][phys, 0, :, slot]
    v = s["pool"].view(-1, 2, hkv, hd, BLOCK)[phys, 1, :, :, slot]
    _store(s["codes"], s["expo"], to, slot, k.double(), v.double())
    _read_back(s["codes"], s["expo"], s["table8"], s["restored"], s["back"], s["ranges"], s["max_len"])
    return s["restored"]


def _softmax_of(s, sc, seen, at, p):
    """Probabilities of scores [.., rows, positions] with the positions `at`, of rows at p, that are seen; rows without one have none."""
    if s["cap"]:
        sc = s["cap"] * torch.tanh(sc / s["cap"])
    if s["slopes"] is not None:
        sc = sc + s["slopes"][:, None, None] * (at - p)
    sc = sc.masked_fill(~seen, -math.inf)
    top = sc.amax(-1, keepdim=True)
    e = torch.exp(sc - torch.where(top > -math.inf, top, 0.0))
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total > 0, total, 1.0)


def _dense(s, phys):
    """Keys [.., Hkv, n, hd] and values [.., Hkv, hd, n] of blocks phys [.., blocks], in float32."""
    hkv, hd = s["hkv"], s["hd"]
    unit = _power(s["expo"][phys]).float()      # [.., blocks, 2, hkv, 16]
    keys = s["codes"][phys, 0] * unit[..., 0, :, :, None]
    vals = s["codes"].view(-1, 2, hkv, hd, BLOCK)[phys, 1] * unit[..., 1, :, None, :]
    return keys.transpose(-4, -3).flatten(-3, -2), vals.movedim(-4, -2).flatten(-2, -1)


def _plain_decode(s):
    h, hkv, hd, t = s["h"], s["hkv"], s["hd"], s["q"].shape[0]
    ctx = s["ctx"].long()
    first = s["first"].long() if s["first"] is not None else torch.zeros_like(ctx)
    if s["window"]:
        first = torch.maximum(first, ctx - s["window"])
    nb = -(-s["max_ctx"] // BLOCK)
    keys, vals = _dense(s, s["table"][s["slot"].long(), :nb].long().clamp(min=0))
    q = s["q"].view(t, hkv, h // hkv, hd)
    sc = (q @ keys.transpose(-1, -2).contiguous()) / math.sqrt(hd)      # [t, hkv, g, positions]
    at = torch.arange(nb * BLOCK, device="cuda")
    seen = ((at >= first[:, None]) & (at < ctx[:, None]))[:, None, None]
    p = _softmax_of(s, sc.reshape(t, h, 1, -1), seen, at, (ctx - 1)[:, None, None, None])
    p = p.view(t, hkv, h // hkv, -1)
    return (vals @ p.transpose(-1, -2).contiguous()).transpose(-1, -2).reshape(t, h, hd)


def _plain_prefill(s):
    h, hkv, hd = s["h"], s["hkv"], s["hd"]
    n, before, first, prefix = (torch.as_tensor(v, device="cuda") for v in s["seqs"])
    most, end = max(s["seqs"][0]), s["max_pos"] + 1
    nb = -(-end // BLOCK)
    row = torch.arange(most, device="cuda")
    real = row < n[:, None]      # the sequences' rows, filled up to the longest
    q = torch.zeros((len(n), most, h * hd), device="cuda")
    q[real] = s["q"]
    q = q.view(len(n), most, hkv, h // hkv, hd).permute(0, 2, 3, 1, 4).reshape(len(n), hkv, -1, hd)
    keys, vals = _dense(s, s["table"][:, :nb].long().clamp(min=0))
    sc = (q @ keys.transpose(-1, -2).contiguous()) / math.sqrt(hd)
    at = torch.arange(nb * BLOCK, device="cuda")
    p = (before[:, None] + row)[:, None, :, None]      # [seqs, 1, rows, 1]
    lo = first[:, None, None, None].expand_as(p)
    if s["window"]:
        lo = torch.maximum(lo, p - s["window"] + 1)
    seen = (at >= lo) & (at <= torch.maximum(p, prefix[:, None, None, None] - 1))
    w = _softmax_of(s, sc.view(len(n), h, most, -1), seen, at, p).view(len(n), hkv, -1, nb * BLOCK)
    out = w @ vals.transpose(-1, -2).contiguous()
    return out.view(len(n), h, most, hd).transpose(1, 2)[real]


# ---------------------------------------------------------------- one pass

def run(s):
    if not own:
        return {"write": _plain_write, "move": _plain_move, "decode": _plain_decode, "prefill": _plain_prefill}[s["op"]](s)
    import paper_2406_00059_amd as ld
    if s["op"] == "write":
        if s["scaling"]:
            ld.ldk_rope_table_scaled(s["pos"], s["rot"], s["base"], s["cos_sin"], **s["scaling"])
        ld.ldk_rope_kv_write_q8(s["qkv"], s["cos_sin"], s["pos"], s["slot"], s["table"], s["codes"], s["expo"], s["h"], s["hkv"], s["hd"], s["q"],
                                rot=s["rot"], interleaved=s["interleaved"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS)
        ld.ldk_kv_from_q8(s["codes"], s["expo"], s["table"], s["pool"], s["table"], s["ranges"], s["max_len"], s["hkv"], s["hd"])
        return s["q"], s["pool"]
    if s["op"] == "move":
        ld.ldk_kv_to_q8(s["pool"], s["table"], s["codes"], s["expo"], s["table8"], s["ranges"], s["max_len"], s["hkv"], s["hd"])
        ld.ldk_kv_from_q8(s["codes"], s["expo"], s["table8"], s["restored"], s["back"], s["ranges"], s["max_len"], s["hkv"], s["hd"])
        return s["restored"]
    if s["op"] == "decode":
        ld.ldk_paged_attention_q8(s["q"], s["h"] * s["hd"], s["codes"], s["expo"], s["table"], s["slot"], s["ctx"], s["max_ctx"], s["h"], s["hkv"],
                                  s["hd"], s["out"], s["scratch"], window=s["window"], first=s["first"], softcap=s["cap"], slopes=s["slopes"])
        return s["out"]
    ld.ldk_prefill_attention_q8(s["q"], s["h"] * s["hd"], s["codes"], s["expo"], s["table"], s["tiles"], s["h"], s["hkv"], s["hd"], s["out"],
                                s["max_pos"], window=s["window"], softcap=s["cap"], slopes=s["slopes"], scratch=s["scratch"])
    return s["out"]


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    sh = SHAPES[case["shape"]]
    el = 4 if sh.dtype == "f32" else 2
    h, hkv, hd = sh.n_heads, sh.n_kv_heads, sh.head_dim
    held, full = 2 * hkv * (hd + 1), 2 * hkv * hd * el      # bytes of a position, in 8 bits and in the model's type
    if case["op"] == "write":      # the 8-bit positions are written, and read back into the model's type
        t = case["chunks"] * case["chunk"] + case["singles"]
        return {"bytes": t * (4 * (2 * h + 2 * hkv) * hd + 4 * case["rot"] + 2 * held + full), "flops": t * (h + 2 * hkv) * hd * 10}
    if case["op"] == "move":
        n = sum(_lengths(case["seqs"], case["len_lo"], case["len_hi"]))
        return {"bytes": n * 2 * (held + full), "flops": n * 2 * hkv * hd * 4}
    w = case["window"]
    if case["op"] == "decode":
        ctx = _contexts(case)
        seen = sum(max(0, c - max(f, c - w if w else 0)) for c, f in zip(ctx, _starts(case, ctx)))
        return {"bytes": seen * held + len(ctx) * 8 * h * hd, "flops": seen * h * hd * 4}
    nbytes, flops = 0, 0
    for n, before, first, prefix in zip(*_segments(case)):
        p = np.arange(before, before + n)
        lo = np.maximum(first, p - w + 1) if w else np.full(n, first)
        hi = np.maximum(p, prefix - 1)
        nbytes += (hi.max() + 1 - lo.min()) * held + n * 8 * h * hd
        flops += int((hi + 1 - lo).sum()) * h * hd * 4
    return {"bytes": int(nbytes), "flops": flops}


# ---------------------------------------------------------------- the definitions in 64 bits

def _value(x):
    """What vectors [.., hd] (float64, on the host) stand for in 8 bits."""
    top = np.abs(x).max(-1)
    unit = np.exp2(np.maximum(np.floor(np.log2(np.where(top > 0, top, 1.0))) - 6, -126.0))[..., None]
    return np.clip(np.rint(x / unit), -127, 127) * unit


def _exact_write(s):
    """Pairs as complex numbers, one row after another."""
    h, hkv, hd, rot = s["h"], s["hkv"], s["hd"], s["rot"]
    x = s["qkv"].double().cpu().numpy().reshape(-1, h + 2 * hkv, hd)
    pos, slot, table = s["pos"].tolist(), s["slot"].tolist(), s["table"].cpu().numpy()
    q, pool = np.zeros((len(pos), h, hd)), np.zeros(tuple(s["pool"].shape))
    vals = pool.reshape(-1, 2, hkv, hd, BLOCK)
    i = np.arange(rot // 2)
    one, two = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + rot // 2)
    table_of = s["cos_sin"].double().cpu().numpy()
    if s["scaling"]:
        c, freq = s["scaling"], 1.0 / float(s["base"]) ** (2.0 * i / rot)
        turns = c["original"] * freq / (2 * np.pi)
        keep = np.clip((turns - c["low"]) / (c["high"] - c["low"]), 0, 1)
        freq, size = (1 - keep) * freq / c["factor"] + keep * freq, float(np.float32(c["attention"]))
    for t, p in enumerate(pos):
        heads = x[t, :h + hkv].copy()
        if s["q_gain"] is not None:
            heads /= np.sqrt((heads ** 2).mean(-1, keepdims=True) + float(np.float32(EPS)))
            heads[:h] *= s["q_gain"].double().cpu().numpy()
            heads[h:] *= s["k_gain"].double().cpu().numpy()
        turn = table_of[t, :, 0] + 1j * table_of[t, :, 1]
        if s["scaling"]:      # the table is in float32
            turn = (size * np.exp(1j * p * freq)).astype(np.complex64).astype(np.complex128)
        z = (heads[:, one] + 1j * heads[:, two]) * turn
        heads[:, one], heads[:, two] = z.real, z.imag
        q[t] = heads[:h]
        b = table[slot[t], p // BLOCK]
        pool[b, 0, :, p % BLOCK] = _value(heads[h:])
        vals[b, 1, :, :, p % BLOCK] = _value(x[t, h + hkv:])
    return torch.from_numpy(q.reshape(len(pos), h * hd)), torch.from_numpy(pool)


def _exact_move(s):
    hkv, hd = s["hkv"], s["hd"]
    out = torch.zeros(tuple(s["restored"].shape), dtype=torch.float64)
    table, back = s["table"].cpu(), s["back"].cpu()
    for seq, first, end in s["ranges"].tolist():
        for b in range(-(-end // BLOCK)):
            n = min(BLOCK, end - b * BLOCK)
            src, dst = s["pool"][table[seq, b]].double().cpu().numpy(), out[back[seq, b]].numpy()
            dst[0, :, :n] = _value(src[0])[:, :n]
            dst[1].reshape(hkv, hd, BLOCK)[:, :, :n] = _value(src[1].reshape(hkv, hd, BLOCK).swapaxes(1, 2)).swapaxes(1, 2)[:, :, :n]
    return out


def _exact_rows(s, q, seq, p, lo, hi):
    """Attention of rows q [n, h, hd] of one sequence, row i over positions lo[i] .. hi[i] of it, head by head."""
    h, hkv, hd = s["h"], s["hkv"], s["hd"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    end = int(hi.max()) + 1
    if end <= 0:
        return out
    blocks = s["table"][seq, :-(-end // BLOCK)].long()
    two = torch.tensor(2.0, dtype=torch.float64, device="cuda")
    at = torch.arange(end, device="cuda")
    seen = (at >= lo[:, None]) & (at <= hi[:, None])
    for j in range(hkv):
        e = s["expo"][blocks][:, :, j].double()
        k = (s["codes"][blocks, 0, j].double() * torch.pow(two, e[:, 0])[..., None]).reshape(-1, hd)[:end]
        v = s["codes"][blocks, 1, j].reshape(-1, hd, BLOCK).transpose(1, 2).double() * torch.pow(two, e[:, 1])[..., None]
        v = v.reshape(-1, hd)[:end].contiguous()
        for i in range(j * (h // hkv), (j + 1) * (h // hkv)):
            sc = torch.mm(q[:, i].double(), k.t().contiguous()) * hd ** -0.5
            if s["cap"]:
                x = torch.exp(-2 * sc.abs() / s["cap"])
                sc = torch.sign(sc) * s["cap"] * (-torch.expm1(-2 * sc.abs() / s["cap"])) / (1 + x)
            if s["slopes"] is not None:
                sc = sc + s["slopes"][i].double() * (at - p[:, None])
            sc = torch.where(seen, sc, -math.inf)
            w = torch.softmax(sc, 1).nan_to_num(0.0)      # a row without a position
            out[:, i] = torch.mm(w, v)
    return out


def exact(case, seed):
    """What run() returns, from the definitions in 64 bits."""
    s = prepare(case, seed)
    if s["op"] == "write":
        return _exact_write(s)
    if s["op"] == "move":
        return _exact_move(s)
    w = s["window"]
    if s["op"] == "decode":
        q, ctx = s["q"].view(-1, s["h"], s["hd"]), s["ctx"].long()
        lo = s["first"].long() if s["first"] is not None else torch.zeros_like(ctx)
        lo = torch.maximum(lo, ctx - w) if w else lo
        return torch.cat([_exact_rows(s, q[t:t + 1], t, ctx[t:t + 1] - 1, lo[t:t + 1], ctx[t:t + 1] - 1) for t in range(len(ctx))])
    out, at = [], 0
    for seq, (n, before, first, prefix) in enumerate(zip(*s["seqs"])):
        p = torch.arange(before, before + n, device="cuda")
        lo = (p - w + 1).clamp(min=first) if w else torch.full_like(p, first)
        out.append(_exact_rows(s, s["q"][at:at + n].view(n, s["h"], s["hd"]), seq, p, lo, p.clamp(min=prefix - 1)))
        at += n
    return torch.cat(out)
