"""A reasoning trace longer than its key/value cache: two models on 4-bit caches, with the operators around them in the order of the method.

A small model writes; at the end of each of its segments a large one catches up on what it has not seen (one pass over several new rows), writes
a few tokens and hands back.  A cache that has no room for the next pass is cut back to `budget` tokens a sequence: every kv head drops the tokens that
received the least attention so far.  Weights and token embeddings are random, so the trace says nothing; its shapes are a model's.

    python -m paper_2504_12329_amd.kv4_trace --small qwen1p5b --large qwen32b --layers 8 --prompt 512 --tokens 2048 --budget 1024
"""
import argparse

import torch
import torch.nn.functional as F

from . import binding as B
from . import synth
from .defaults import N1, N2


class Context:
    """A decoder whose attention runs on a 4-bit cache, for several sequences of equal or unequal length.

    Between calls it holds what the cache's calls want to be told: the slots each sequence has, and the position it is at."""

    def __init__(self, model, seed, n_seq, max_pos, budget, recent, max_rows, n_layers=None):
        self.cfg = synth.model_config(model, max_pos, n_layers=n_layers)
        self.budget, self.recent, self.max_rows = budget, recent, max_rows
        shape = {n: self.cfg[n] for n in ("n_layers", "n_q_heads", "n_kv_heads", "head_dim", "rms_eps")}
        self.kv = B.Kv4Cache(dict(shape, n_seq=n_seq, max_seq=budget + max_rows, max_rows=n_seq * max_rows, max_pos=max_pos),
                             B.rope_table(max_pos, self.cfg["head_dim"], self.cfg["rope_theta"]))
        slots = (self.cfg["n_layers"], n_seq, self.cfg["n_kv_heads"], budget + max_rows)
        self.ledger = B.Kv4Ledger(torch.zeros(slots, device="cuda"), torch.zeros(slots, dtype=torch.int32, device="cuda"))
        self.layers = [synth.make_layer(self.cfg, seed, i, device="cuda") for i in range(self.cfg["n_layers"])]
        self.slots, self.pos = [0] * n_seq, [0] * n_seq
        self.evictions = 0

    def forward(self, x, rows):
        """New rows, rows[s] of sequence s one after the other: x bf16 [sum(rows)][hidden].  Returns the last layer's output."""
        self._make_room(rows)
        spans = B.Kv4Spans([(s, self.slots[s], self.pos[s], r) for s, r in enumerate(rows)])
        h = self.cfg["hidden"]
        for i, w in enumerate(self.layers):
            y = F.rms_norm(x, (h,), w["norm_attn"], self.cfg["rms_eps"])
            q = self.kv.append(i, spans, F.linear(y, w["wqkv"], w["bqkv"]), ledger=self.ledger)
            a = self.kv.attend(i, spans, q, self.ledger)
            x = x + F.linear(a.flatten(1), w["wo"])
            gate, up = F.linear(F.rms_norm(x, (h,), w["norm_mlp"], self.cfg["rms_eps"]), w["w_gate_up"]).chunk(2, -1)
            x = x + F.linear(F.silu(gate) * up, w["w_down"])
        for s, r in enumerate(rows):
            self.slots[s] += r
            self.pos[s] += r
        return x

    def _make_room(self, rows):
        if all(n + r <= self.budget + self.max_rows for n, r in zip(self.slots, rows)):
            return
        over = B.Kv4Spans([(s, n, self.pos[s], 0) for s, n in enumerate(self.slots) if n > self.budget])
        self.kv.evict(0, self.cfg["n_layers"], over, self.budget, self.recent, self.ledger)
        self.slots = [min(n, self.budget) for n in self.slots]
        self.evictions += 1

    def prefill(self, x, rows):
        """forward() in passes of at most max_rows rows of each sequence.  Returns the outputs of all rows, in the order of x."""
        parts, passes = x.split(rows), []
        for at in range(0, max(rows), self.max_rows):
            now = [p[at:at + self.max_rows] for p in parts]
            passes.append(self.forward(torch.cat(now), [len(p) for p in now]).split([len(p) for p in now]))
        return torch.cat([p[s] for s in range(len(rows)) for p in passes]) if passes else x


def trace(small, large, n_seq, prompt, tokens, seed=0, segment=N2, takeover=N1):
    """Prompt into the small model; then segments it writes alone, each followed by a takeover of the large one.  Token embeddings are
    drawn at random.  Returns the tokens written by each and the models' last outputs."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def embed(model, rows):
        return torch.randn(rows, model.cfg["hidden"], dtype=torch.bfloat16, device="cuda", generator=gen)

    wrote, out = {"small": 0, "large": 0}, {}
    unread = {"small": 0, "large": prompt}              # tokens of the trace that a model has not read yet
    out["small"] = small.prefill(embed(small, n_seq * prompt), [prompt] * n_seq)
    while wrote["small"] + wrote["large"] < tokens:
        for name, model, most in (("small", small, segment), ("large", large, takeover)):
            n = min(most, tokens - wrote["small"] - wrote["large"])
            if not n:
                break
            if unread[name]:                             # catch up on the other's tokens
                out[name] = model.prefill(embed(model, n_seq * unread[name]), [unread[name]] * n_seq)
                unread[name] = 0
            for _ in range(n):
                out[name] = model.forward(embed(model, n_seq), [1] * n_seq)
            wrote[name] += n
            unread["large" if name == "small" else "small"] += n
    return wrote, out


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--small", default="qwen1p5b", choices=synth.SHAPES)
    ap.add_argument("--large", default="qwen7b", choices=synth.SHAPES)
    ap.add_argument("--layers", type=int, default=4, help="layers of each model (0: all)")
    ap.add_argument("--sequences", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=512)
    ap.add_argument("--tokens", type=int, default=1024)
    ap.add_argument("--budget", type=int, default=768)
    ap.add_argument("--recent", type=int, default=128)
    ap.add_argument("--rows", type=int, default=256, help="most rows of a sequence in one pass")
    a = ap.parse_args(argv)
    models = [Context(m, i, a.sequences, a.prompt + a.tokens, a.budget, a.recent, a.rows, a.layers or None)
              for i, m in enumerate((a.small, a.large))]
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    trace(*models, a.sequences, a.prompt, min(a.tokens, 2))     # warm up
    for m in models:
        m.slots, m.pos, m.evictions = [0] * a.sequences, [0] * a.sequences, 0
    start.record()
    wrote, _ = trace(*models, a.sequences, a.prompt, a.tokens)
    end.record()
    end.synchronize()
    print(f"{a.sequences} sequences, prompt of {a.prompt}, {wrote['small']} + {wrote['large']} tokens each: {start.elapsed_time(end):.0f} ms")
    for name, m in zip((a.small, a.large), models):
        c = m.cfg
        numbers = 2 * c["n_layers"] * a.sequences * c["n_kv_heads"] * c["head_dim"]
        print(f"{name}, {c['n_layers']} layers: at position {m.pos[0]} with {m.slots[0]} slots after {m.evictions} evictions; cache "
              f"{m.kv.cache.numel() / 1e6:.1f} MB, all positions in bf16 {2 * numbers * max(m.pos[0], 1) / 1e6:.1f} MB")


if __name__ == "__main__":
    main()
