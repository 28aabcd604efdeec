"""A decoder that reads few bytes a step: 4-bit weights, attention over the cache blocks that matter, tokens chosen under rules.

The engine's calls (ld_prefill, ld_decode_step, ..) stream every bf16 matrix and every sequence's whole cache.  A
LightDecoder runs the same decoder on the same paged cache with the kernel-level operators for that: ldk_linear_w4 for
all matrices, ldk_kv_summary + ldk_sparse_attention for decode rows (prompt rows attend to everything before them), and
ldk_choose, which keeps a tool call inside its grammar.  Blocks, sequences and positions are the KV object's: sequences are allocated, freed,
swapped and forked there, and refresh() takes over one whose blocks were not filled here or have moved since.

    light = LightDecoder(model, kv, budget=64)
    seq = ld_kv_alloc(kv.h)
    light.prefill(seq, prompt)
    for _ in range(n):
        tokens = light.step([seq], mask=grammar_mask)
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding as ld


class LightDecoder:
    """model: a Model whose matrices are quantised here (its own stay as they are and may be dropped by the caller); kv: a KV
    of that model.  group, zeros: of the 4-bit weights.  budget, keep_first, keep_last: blocks of 16 positions a decode row
    attends to per KV head.  max_rows: rows of a pass (longer prompts go in chunks).  penalties: (repetition, presence, frequency)."""

    def __init__(self, model, kv, group=128, zeros=False, budget=64, keep_first=1, keep_last=4, max_rows=256, penalties=None, device="cuda"):
        sh = model.shape
        self.shape, self.kv, self.device = sh, kv, device
        self.budget, self.keep_first, self.keep_last, self.max_rows = budget, keep_first, keep_last, max_rows
        st = torch.bfloat16 if sh.dtype == "bf16" else torch.float32
        w = model.weights

        def quantise(m, parts=1):
            return ld.W4Matrix.quantize(m, group, parts, st, zeros)
        self.wqkv = [quantise(m) for m in w["wqkv"]]
        self.wo = [quantise(m) for m in w["wo"]]
        self.wgate_up = [quantise(m, 2) for m in w["wgate_up"]]
        self.wdown = [quantise(m) for m in w["wdown"]]
        self.lm_head = quantise(w["lm_head"])
        self.embed, self.attn_norm, self.ffn_norm, self.final_norm = w["embed"], w["attn_norm"], w["ffn_norm"], w["final_norm"]

        hd, T, L = sh.head_dim, max_rows, sh.n_layers
        self.nq, self.nqkv = sh.n_heads * hd, (sh.n_heads + 2 * sh.n_kv_heads) * hd
        f = dict(dtype=torch.float32, device=device)
        self.x, self.qkv = torch.empty((T, sh.d_model), **f), torch.empty((T, self.nqkv), **f)
        self.att, self.act = torch.empty((T, sh.n_heads, hd), **f), torch.empty((T, sh.d_ffn), **f)
        self.cos_sin, self.logits = torch.empty((T, hd // 2, 2), **f), torch.empty((T, sh.vocab), **f)
        self.bounds = torch.zeros((L, kv.n_blocks, sh.n_kv_heads, 2, hd), dtype=torch.int8, device=device)
        self.unit = torch.ones((L, kv.n_blocks, sh.n_kv_heads), **f)
        self.sel = torch.empty((T, sh.n_kv_heads, budget), dtype=torch.int32, device=device)
        max_ctx = kv.max_blocks * sh.kv_block
        shapes = [(self.nqkv, sh.d_model, ld.LDK_STORE), (sh.d_model, self.nq, ld.LDK_ADD), (sh.d_ffn, sh.d_model, ld.LDK_SWIGLU),
                  (sh.d_model, sh.d_ffn, ld.LDK_ADD), (sh.vocab, sh.d_model, ld.LDK_STORE)]
        need = max(ld.ldk_linear_w4_scratch_bytes(T, n, k, e) for n, k, e in shapes)
        need = max(need, ld.ldk_sparse_attention_scratch_bytes(T, sh.n_heads, sh.n_kv_heads, hd, max_ctx, sh.window, budget),
                   max(ld.ldk_attention_scratch_bytes(t, sh.n_heads, sh.n_kv_heads, hd, max_ctx, sh.window) for t in range(1, T + 1)),
                   ld.ldk_prefill_attention_scratch_bytes(), ld.ldk_choose_scratch_bytes(T, sh.vocab))
        self.scratch = torch.empty(need, dtype=torch.uint8, device=device)

        # block tables and token histories of every sequence, on the device
        n_seqs = kv.max_seqs
        self.table = torch.full((n_seqs, kv.max_blocks), -1, dtype=torch.int32, device=device)
        self.history = torch.zeros((n_seqs, max_ctx + 1), dtype=torch.int32, device=device)
        self.length = [0] * n_seqs           # tokens of the history: the cached ones and the pending one
        self.prompt = [0] * n_seqs
        self.generation = [0] * n_seqs       # of the blocks that table and bounds are of
        self.penalties = None if penalties is None else torch.tensor([penalties] * T, **f)

    def _i32(self, v):
        return torch.as_tensor(np.ascontiguousarray(v, dtype=np.int32)).to(self.device)

    def _tokens(self, v):
        """Token ids as an int32 array; the embedding is read by them."""
        a = np.asarray(v)
        if a.size == 0:
            return np.empty(0, np.int32)
        if a.ndim != 1 or a.dtype.kind not in "iu" or a.min() < 0 or a.max() >= self.shape.vocab:
            raise ValueError(f"tokens have to be a sequence of whole numbers in 0 .. {self.shape.vocab - 1}")
        return a.astype(np.int32)

    def _map(self, seq, n_tokens):
        """Maps the next n_tokens positions of a sequence and brings the device's copy of its block table up to date."""
        first = ld.ld_kv_len(self.kv.h, seq)
        ld.ld_kv_assume(self.kv.h, seq, n_tokens)
        if first % 16 == 0 or first % 16 + n_tokens > 16:
            t = ld.ld_kv_block_table(self.kv.h, seq)
            self.table[seq, :t.size] = self._i32(t)
        return first

    def _check_own(self, seq, new=False):
        """Raises where the sequence holds blocks that the decoder has not filled or been shown (table and bounds are of others); new: it may hold none."""
        if not 0 <= seq < len(self.length) or ld.ld_kv_len(self.kv.h, seq) < 0:
            raise ValueError(f"no sequence {seq}")
        if self.generation[seq] != ld.ld_kv_generation(self.kv.h, seq) and not (new and ld.ld_kv_len(self.kv.h, seq) == 0):
            raise ValueError(f"the blocks of sequence {seq} were replaced (freed, forked or swapped): refresh it first")

    RULES = ("bias_start", "bias_token", "bias", "mask", "mask_row", "temperature", "seed")

    def _check_rules(self, R, rules):
        """Raises what _choose for R rows would refuse, before anything is fed."""
        if not rules:
            return
        for name in rules:
            if name not in self.RULES:
                raise TypeError(f"no rule is named {name} (histories, positions and penalties are the decoder's own)")
        ld.ldk_choose(self.logits[:R], self.sel.view(-1)[:R], check_only=True, stream=0, **rules)
        given = {name for name in rules if rules[name] is not None}
        if "temperature" in given and "seed" not in given:
            raise ld.LdError(ld.LD_E_INVAL, "a temperature needs a seed")
        if given & {"bias", "bias_start", "bias_token"} and not {"bias", "bias_start", "bias_token"} <= given:
            raise ld.LdError(ld.LD_E_INVAL, "bias comes with bias_start and bias_token")
        if "mask" in given and "mask_row" not in given and rules["mask"].shape[0] < R:
            raise ld.LdError(ld.LD_E_INVAL, f"a mask of {R} rows, or a mask_row for each of the {R} sequences")

    def _check_room(self, seqs):
        """Raises what _map of one position for each of these sequences would end in, before any of them is mapped."""
        need = 0
        for s in seqs:
            n = ld.ld_kv_len(self.kv.h, s)
            if n // 16 >= self.kv.max_blocks:
                raise ld.LdError(ld.LD_E_RANGE, f"sequence {s} is as long as its block table allows")
            if n % 16 == 0:
                t = ld.ld_kv_block_table(self.kv.h, s, self.kv.max_blocks)
                need += n // 16 >= t.size or t[n // 16] < 0
        if need > ld.ld_kv_free_blocks(self.kv.h):
            raise ld.LdError(ld.LD_E_NOMEM, "out of KV blocks")

    def _pass(self, tok, seqs, first, count, decode):
        """Rows of sequences seqs (count[i] rows each from position first[i]) through all layers; the residual stream is left in x."""
        sh, h, hkv, hd = self.shape, self.shape.n_heads, self.shape.n_kv_heads, self.shape.head_dim
        pos = np.concatenate([np.arange(f, f + n) for f, n in zip(first, count)])
        slot = np.repeat(np.asarray(seqs), count)
        T, max_ctx = len(pos), int(pos.max()) + 1
        d_pos, d_slot, d_ctx = self._i32(pos), self._i32(slot), self._i32(pos + 1)
        ranges = self._i32(np.stack([seqs, first, np.add(first, count)], 1))
        x, qkv, att, act, cs = self.x[:T], self.qkv[:T], self.att[:T], self.act[:T], self.cos_sin[:T]
        tiles = None
        if not decode and sh.dtype == "bf16" and hd == 128:      # chunk attention takes up to 128 rows of a sequence a tile
            rows, at = [], 0
            for s, f, n in zip(seqs, first, count):
                rows += [(at + i, min(128, n - i), f + i, s) for i in range(0, n, 128)]
                at += n
            tiles = self._i32(np.array(rows))
        ld.ldk_embed(self.embed, tok, x)
        ld.ldk_rope_table(d_pos, hd, sh.rope_base, cs)
        for l in range(sh.n_layers):
            pool = self.kv.pool[l]
            ld.ldk_linear_w4(self.wqkv[l], x, qkv, g=self.attn_norm[l], eps=sh.rms_eps, scratch=self.scratch)
            ld.ldk_rope_kv_write(qkv, cs, d_pos, d_slot, self.table, pool, h, hkv, hd)
            ld.ldk_kv_summary(pool, self.table, ranges, max(count), hkv, hd, self.bounds[l], self.unit[l])
            if decode:
                ld.ldk_sparse_attention(qkv, self.nqkv, pool, self.bounds[l], self.unit[l], self.table, d_slot, d_ctx, max_ctx, h, hkv, hd, self.budget,
                                        self.keep_first, self.keep_last, att, self.sel[:T], self.scratch, window=sh.window)
            elif tiles is not None:
                ld.ldk_prefill_attention(qkv, self.nqkv, pool, self.table, tiles, h, hkv, hd, att, max_ctx - 1, window=sh.window, scratch=self.scratch)
            else:
                ld.ldk_paged_attention(qkv, self.nqkv, pool, self.table, d_slot, d_ctx, max_ctx, h, hkv, hd, att, self.scratch, window=sh.window)
            ld.ldk_linear_w4(self.wo[l], att.view(T, self.nq), x, ld.LDK_ADD, scratch=self.scratch)
            ld.ldk_linear_w4(self.wgate_up[l], x, act, ld.LDK_SWIGLU, g=self.ffn_norm[l], eps=sh.rms_eps, scratch=self.scratch)
            ld.ldk_linear_w4(self.wdown[l], act, x, ld.LDK_ADD, scratch=self.scratch)
        return x

    def _choose(self, x, seqs, rules):
        """Logits of the rows of x and one token each, which becomes the sequence's pending one; -1 and none where the rules leave no token."""
        R = x.shape[0]
        logits, token = self.logits[:R], torch.empty(R, dtype=torch.int32, device=self.device)
        ld.ldk_linear_w4(self.lm_head, x, logits, g=self.final_norm, eps=self.shape.rms_eps, scratch=self.scratch)
        rows = self._i32(seqs).long()
        length = self._i32([self.length[s] for s in seqs])
        if self.penalties is not None:
            rules = dict(rules, history=self.history[rows], history_len=length, n_prompt=self._i32([self.prompt[s] for s in seqs]),
                         penalties=self.penalties[:R])
        if rules.get("temperature") is not None:
            rules = dict(rules, pos=length)
        ld.ldk_choose(logits, token, scratch=self.scratch, **rules)
        self.history[rows, length.long()] = token      # behind the end of a row that gets no token
        token = token.tolist()
        for s, t in zip(seqs, token):
            if t >= 0:
                self.length[s] += 1
                ld.ld_kv_assume(self.kv.h, s, 0, t)      # the engine's pending token (none since _map), should it carry the sequence on
        return token

    def prefill(self, seq, tokens, **rules):
        """Feeds [pending?] ++ tokens and returns the token chosen after the last one.  rules: as in step."""
        tokens = self._tokens(tokens)
        self._check_own(seq, new=True)
        first = ld.ld_kv_len(self.kv.h, seq)
        at = self.length[seq] if self.generation[seq] == ld.ld_kv_generation(self.kv.h, seq) else 0      # else a new sequence
        if not first <= at <= first + 1:
            raise ValueError(f"prefill: sequence {seq} has positions that were fed elsewhere (refresh it first)")
        if at + tokens.size <= first:
            raise ValueError("prefill: no token to feed")
        self._check_rules(1, rules)
        self._map(seq, at + tokens.size - first)      # of the whole prompt: a shortage changes nothing
        self.history[seq, at:at + tokens.size] = self._i32(tokens)
        self.length[seq] = self.prompt[seq] = at + tokens.size
        self.generation[seq] = ld.ld_kv_generation(self.kv.h, seq)
        while first < self.length[seq]:
            n = min(self.max_rows, self.length[seq] - first)
            x = self._pass(self.history[seq, first:first + n], [seq], [first], [n], False)[n - 1:n]
            first += n
        return self._choose(x, [seq], rules)[0]

    def refresh(self, seq, tokens=None, pending=None, n_prompt=None):
        """Takes over a sequence whose cached positions were filled elsewhere (by the engine, a fork): its block table, its history (tokens: those of
        the cached positions; pending: the one to be fed next; n_prompt: how many of them are prompt, all cached ones if not given) and the bounds of
        all its blocks.  Without tokens: a sequence that was fed here and has only moved (a swap); its history stays."""
        n, sh = ld.ld_kv_len(self.kv.h, seq), self.shape
        if tokens is None:
            if n < 0 or not n <= self.length[seq] <= n + 1 or pending is not None:
                raise ValueError(f"refresh: the tokens of the {n} cached positions of sequence {seq} are not known here")
            length, n_prompt = self.length[seq], self.prompt[seq] if n_prompt is None else n_prompt
        else:
            tokens = self._tokens(list(tokens) + ([] if pending is None else [pending]))
            length, n_prompt = len(tokens), n if n_prompt is None else n_prompt
            if length != n + (pending is not None):
                raise ValueError(f"refresh: {n} cached positions")
        if not 0 <= n_prompt <= n:
            raise ValueError(f"refresh: a prompt of {n_prompt} of {n} cached tokens")
        t = ld.ld_kv_block_table(self.kv.h, seq)
        if t.size * 16 < n:
            raise ValueError(f"refresh: sequence {seq} is swapped out")
        self.table[seq] = -1
        self.table[seq, :t.size] = self._i32(t)
        if tokens is not None:
            self.history[seq, :length] = self._i32(tokens)
        self.length[seq], self.prompt[seq] = length, n_prompt
        self.generation[seq] = ld.ld_kv_generation(self.kv.h, seq)
        ranges = self._i32([[seq, 0, n]])
        for l in range(sh.n_layers):
            ld.ldk_kv_summary(self.kv.pool[l], self.table, ranges, n, sh.n_kv_heads, sh.head_dim, self.bounds[l], self.unit[l])

    def step(self, seqs, **rules):
        """One decode iteration: feeds every sequence's pending token and returns the tokens chosen after them (-1 where no token is allowed: that
        sequence then has none pending, and goes on with a prefill).  rules: ldk_choose's bias_start,
        bias_token, bias, mask, mask_row, temperature and seed, a row per sequence (the histories are the decoder's own)."""
        if not 0 < len(seqs) <= self.max_rows or len(set(seqs)) != len(seqs):
            raise ValueError(f"step: between one and {self.max_rows} distinct sequences")
        for s in seqs:
            self._check_own(s)
        if any(self.length[s] != ld.ld_kv_len(self.kv.h, s) + 1 for s in seqs):
            raise ValueError("step: a sequence without a pending token (prefill it, or refresh it first)")
        self._check_rules(len(seqs), rules)
        self._check_room(seqs)
        first = [self._map(s, 1) for s in seqs]
        tok = self.history[self._i32(seqs).long(), self._i32(first).long()]
        return self._choose(self._pass(tok, list(seqs), first, [1] * len(first), True), seqs, rules)


def main():
    """A small decoder with seeded weights: a prompt, free tokens, then tokens from a small set only, as inside a tool call's grammar."""
    from workloads import LLAMA7B, make_weights
    sh = LLAMA7B.with_layers(2)
    model = ld.Model(sh, make_weights(sh, 1, device="cuda"))
    kv = ld.KV(model, 600, 64, 2, 300)
    light = LightDecoder(model, kv, budget=16, penalties=(1.1, 0.0, 0.1))
    seq = ld.ld_kv_alloc(kv.h)
    out = [light.prefill(seq, np.arange(4000) * 7919 % sh.vocab)]
    out += [light.step([seq])[0] for _ in range(15)]
    print("free:     ", out)
    mask = torch.zeros((1, sh.vocab // 32), dtype=torch.int32, device="cuda")
    mask[0, 100] = 0b1011
    print("in a mask:", [light.step([seq], mask=mask)[0] for _ in range(8)])


if __name__ == "__main__":
    main()
