"""Decoding with a cache in 8 bits: the target model of a configuration, one token per sequence and step, on the library's kernels.

    python -m paper_2503_01840_b200.kv8_decode [--shape C2] [--layers 4] [--batch 2] [--prompt 700] [--steps 16] [--cache e4m3,int8,bf16]

SpecDecoder keeps its cache in bf16 or fp32.  This is a loop of a program's own around the single operators: projections by
gemm_fused / gemm_wide, gate/up by gemm_swiglu, tokens' rows by embedding, the residual stream's sums and norms by rms_norm, and for the cache
  kv_append         rotates queries and keys, quantises keys and values, writes them to the pages
  kv_read           reads a prompt's keys and values back for its own attention (ttt_attention without simulated steps: plain causal)
  decode_attention  attends from every sequence's new token
Prints a JSON line per cache format: time per step, bytes of the cache per token, and how many tokens equal those of the bf16 cache.
"""
import argparse
import json

import torch

from . import binding as sb
from . import synth

FORMATS = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}


class CachedDecoder:
    """A bf16 target (weights as of synth.make_target_weights) with its own paged cache for `batch` sequences of up to max_ctx positions; a prompt or step beyond
    them is refused.  scaling: arguments of rope_frequencies for contexts longer than the trained one, e.g. dict(scaling="wavelength", factor=8.0)."""

    def __init__(self, cfg, weights, batch: int, max_ctx: int, cache: str = "e4m3", scaling=None):
        self.m, self.w, self.batch, self.max_ctx = cfg, weights, batch, max_ctx
        per_seq = -(-max_ctx // cfg.page_size)
        g = torch.Generator().manual_seed(1)
        self.table = torch.randperm(batch * per_seq, generator=g).view(batch, per_seq).to(torch.int32).cuda()
        shape = (batch * per_seq, cfg.n_kv_heads, cfg.page_size, cfg.head_dim)
        dt = FORMATS[cache]
        pool = lambda: torch.zeros(shape, dtype=torch.uint8, device="cuda").view(dt) if dt.itemsize == 1 else torch.zeros(shape, dtype=dt, device="cuda")
        scale = lambda: torch.zeros(shape[:3], device="cuda") if dt.itemsize == 1 else None
        self.layers = [dict(k_pool=pool(), v_pool=pool(), page_table=self.table, k_scale=scale(), v_scale=scale()) for _ in range(cfg.n_layers)]
        self.freq, self.mscale = sb.rope_frequencies(cfg.head_dim, cfg.rope_theta, **(scaling or {}))
        self.workspace = sb.decode_workspace()
        self.wqkv = [torch.cat([l["wq"], l["wk"], l["wv"]]) for l in weights["layers"]]

    def cache_bytes_per_token(self) -> int:
        return sum(t.nbytes // (t.shape[0] * t.shape[2]) for l in self.layers for n, t in l.items() if t is not None and n != "page_table")

    # -- pieces of a layer
    def _norm(self, x, y, gain):
        """(the norm of the residual stream x with y added in bf16, the stream): y is what the part before has left to add, if any"""
        if y is None:
            return sb.rms_norm(x, gain, self.m.rms_eps, dtype=torch.bfloat16), x
        return sb.rms_norm(y, gain, self.m.rms_eps, residual=x, dtype=torch.bfloat16, sum_out=x)

    def _linear(self, x, w):
        return sb.gemm_fused(x, w) if x.shape[0] <= 128 else sb.gemm_wide(x, w)[0]

    def _mlp(self, x, y, l):
        h, x = self._norm(x, y, l["mlp_norm"])
        act = sb.gemm_swiglu(h, l["w_gate"], l["w_up"]) if h.shape[0] <= 128 else sb.gemm_wide(h, l["w_gate"], l["w_up"])[0]
        return x, self._linear(act, l["w_down"])

    def _layer(self, i, x, y, seq, pos, attend):
        """attend(queries, layer's cache) -> [rows][heads * head_dim]; (x, y) as of _norm"""
        m, l = self.m, self.w["layers"][i]
        h, x = self._norm(x, y, l["attn_norm"])
        qkv = self._linear(h, self.wqkv[i]).bfloat16().view(-1, m.n_heads + 2 * m.n_kv_heads, m.head_dim)
        H, G = m.n_heads, m.n_kv_heads
        q = sb.kv_append(qkv[:, H: H + G], qkv[:, H + G:], row_seq=seq, row_pos=pos, q=qkv[:, :H], inv_freq=self.freq, mscale=self.mscale, **self.layers[i])
        return self._mlp(x, self._linear(attend(q, self.layers[i]).reshape(x.shape[0], -1), l["wo"]), l)

    def _tokens(self, x, y):
        """(greedy tokens int32, final hidden states)"""
        h, _ = self._norm(x, y, self.w["final_norm"])
        return sb.argmax(self._linear(h, self.w["lm_head"])), h

    def _embed(self, tokens):
        """tokens: integers of any type and stride, on the GPU or not"""
        if tokens.dtype not in (torch.int32, torch.int64):
            tokens = tokens.long()
        return sb.embedding(tokens.cuda().contiguous(), self.w["embed"], dtype=torch.float32)

    # -- the loop; weights may be parameters of a module: nothing is recorded for their gradients
    @torch.no_grad()
    def prefill(self, prompts):
        """Prompts (id sequences) one after the other; the first token of each."""
        if len(prompts) != self.batch or not all(1 <= len(p) <= self.max_ctx for p in prompts):
            raise ValueError(f"prefill: {self.batch} prompts of 1 to {self.max_ctx} tokens")
        prompts = [torch.as_tensor(p).long() for p in prompts]
        if not all(bool(((p >= 0) & (p < self.m.vocab)).all()) for p in prompts):      # before anything is written
            raise ValueError(f"prefill: token ids from 0 to {self.m.vocab - 1}")
        first, m, ps = [], self.m, 16
        for b, prompt in enumerate(prompts):
            T = len(prompt)
            seq, pos = torch.full((T,), b, dtype=torch.int32, device="cuda"), torch.arange(T, dtype=torch.int32, device="cuda")
            pages = -(-T // ps)
            order = torch.arange(pages, dtype=torch.int32, device="cuda")

            def attend(q, cache):
                pool = []
                for rows in sb.kv_read(row_seq=seq, row_kvpos=pos, **cache):
                    rows = torch.nn.functional.pad(rows, (0, 0, 0, 0, 0, pages * ps - T))
                    pool.append(rows.view(pages, ps, m.n_kv_heads, m.head_dim).transpose(1, 2).contiguous())
                return sb.ttt_attention(q, *pool, order, None, None)

            x, y = self._embed(prompt), None
            for i in range(m.n_layers):
                x, y = self._layer(i, x, y, seq, pos, attend)
            first.append(self._tokens(x[-1:], y[-1:])[0])
        self.tokens = torch.cat(first)
        self.lengths = torch.tensor([len(p) for p in prompts], dtype=torch.int32, device="cuda")
        self.longest = max(len(p) for p in prompts)                      # known here without asking the GPU
        self.seqs = torch.arange(self.batch, dtype=torch.int32, device="cuda")
        return self.tokens

    @torch.no_grad()
    def step(self):
        """(the next token of every sequence int32 [batch] on the GPU, hidden states); nothing waits for the GPU."""
        if self.longest >= self.max_ctx:
            raise ValueError(f"step: a sequence has the cache's {self.max_ctx} positions")
        self.longest += 1
        pos, seen = self.lengths, self.lengths + 1
        x, y = self._embed(self.tokens), None
        for i in range(self.m.n_layers):
            x, y = self._layer(i, x, y, self.seqs, pos, lambda q, cache: sb.decode_attention(q, lengths=seen, workspace=self.workspace, **cache))
        self.lengths = seen
        self.tokens, hidden = self._tokens(x, y)
        return self.tokens, hidden


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--shape", default="C2", choices=[n for n, c in synth.CONFIGS.items() if c.dtype == "bf16"])
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--batch", type=int, default=2)
    ap.add_argument("--prompt", type=int, default=700)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--cache", default="bf16,e4m3,int8")
    a = ap.parse_args()
    cfg = synth.CONFIGS[a.shape].truncated(a.layers, batch=a.batch)
    w, dw, _, _ = synth.make_structured(cfg, 1.0, device="cuda", residual_scale=1.0)
    d2t = dw["d2t"].cpu()
    prompts = [synth.structured_prompt(cfg, d2t, a.prompt + 37 * b, seed=b) for b in range(a.batch)]
    want = None
    for name in ["bf16"] + [n for n in a.cache.split(",") if n != "bf16"]:
        dec = CachedDecoder(cfg, w, a.batch, a.prompt + 37 * a.batch + a.steps, name)
        got = [dec.prefill(prompts)]
        got += [dec.step()[0] for _ in range(3)]
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        got += [dec.step()[0] for _ in range(a.steps - 3)]
        e1.record()
        torch.cuda.synchronize()
        got = torch.stack(got)
        want = got if want is None else want
        print(json.dumps({"cache": name, "shape": a.shape, "layers": a.layers, "batch": a.batch, "prompt": a.prompt, "cache_bytes_per_token": dec.cache_bytes_per_token(),
                          "ms_per_step": round(e0.elapsed_time(e1) / max(1, a.steps - 3), 4), "tokens_as_bf16": int((got == want).sum()), "tokens": got.numel()}), flush=True)


if __name__ == "__main__":
    main()
