"""Drafts by a small model, verified by a large one, on caches in pages: the comparison system of the method this library is for, with the operators
around its passes in order.

In a round the small model writes a tree of tokens after the last decided one (`widths` tokens after each of its rows, level by level); the large one
reads the whole tree in one pass, the verdict keeps a branch of it and draws the token that follows, and the keys and values of that branch are
brought together.  The small model then catches up on what it has not read.  Weights are random unless they are given, so the text says nothing; its shapes are a model's.

    python -m paper_2504_12329_amd.draft_trace --small qwen7b --large qwen32b --layers 4 --prompt 512 --tokens 64 --widths 3 2 1 1
"""
import argparse

import torch
import torch.nn.functional as F

from . import binding as B
from . import synth


class PagedModel:
    """A decoder whose attention runs on a cache in pages, for several sequences; pages are dealt out as they are needed."""

    def __init__(self, model, seed, n_seq, max_pos, max_rows, n_layers=None, page_size=16, weights=None):
        self.cfg = c = synth.model_config(model, max_pos, n_layers=n_layers)
        max_pages = -(-(max_pos + max_rows) // page_size)
        self.table = torch.full((n_seq, max_pages), -1, dtype=torch.int32, device="cuda")
        self.free, self.held, self.page_size = list(range(n_seq * max_pages)), [0] * n_seq, page_size
        shape = {n: c[n] for n in ("n_layers", "n_q_heads", "n_kv_heads", "head_dim", "rms_eps")}
        self.kv = B.PagedCache(dict(shape, n_seq=n_seq, n_pages=len(self.free), page_size=page_size, max_pages=max_pages, max_rows=n_seq * max_rows, max_pos=max_pos),
                               B.rope_table(max_pos, c["head_dim"], c["rope_theta"]), self.table)
        self.w = weights or synth.make_weights(c, seed, device="cuda")
        self.max_rows = max_rows
        self.len = [0] * n_seq                                # tokens whose keys and values are held

    def _make_room(self, spans):
        for seq, length, _, rows in spans:
            while self.held[seq] * self.page_size < length + rows:
                self.table[seq, self.held[seq]] = self.free.pop()
                self.held[seq] += 1

    def forward(self, tokens, spans):
        """Logits after every row, float32 [rows][vocab]; tokens: int [rows] on the GPU."""
        self._make_room(spans.spans)
        h, eps = self.cfg["hidden"], self.cfg["rms_eps"]
        x = self.w["embed"][tokens.long()]
        for i, w in enumerate(self.w["layers"]):
            q = self.kv.append(i, spans, F.linear(F.rms_norm(x, (h,), w["norm_attn"], eps), w["wqkv"], w["bqkv"]))
            x = x + F.linear(self.kv.attend(i, spans, q).flatten(1), w["wo"])
            gate, up = F.linear(F.rms_norm(x, (h,), w["norm_mlp"], eps), w["w_gate_up"]).chunk(2, -1)
            x = x + F.linear(F.silu(gate) * up, w["w_down"])
        head = self.w["embed"] if self.w["lm_head"] is None else self.w["lm_head"]
        return F.linear(F.rms_norm(x, (h,), self.w["final_norm"], eps), head).float()

    def read(self, texts, upto):
        """Feeds texts[s][len[s]:upto[s]], in passes of at most max_rows rows of a sequence.  Nothing comes back."""
        while any(n < u for n, u in zip(self.len, upto)):
            rows = [min(self.max_rows, u - n) for n, u in zip(self.len, upto)]
            spans = B.Kv4Spans([(s, n, n, r) for s, (n, r) in enumerate(zip(self.len, rows))])
            new = [t for s, r in enumerate(rows) for t in texts[s][self.len[s]:self.len[s] + r]]
            self.forward(torch.tensor(new, device="cuda"), spans)
            self.len = [n + r for n, r in zip(self.len, rows)]

    def keep(self, spans, path, accepted, counts):
        """After a pass over drafts: the branch that stays, brought together."""
        self.kv.keep(0, self.cfg["n_layers"], spans, path, accepted)
        self.len = [n + 1 + c for n, c in zip(self.len, counts)]


def parents_of(widths):
    """The row that each row of a tree follows: row 0, then widths[0] rows after it, widths[1] after each of those, ...; and the levels' first rows."""
    parents, levels = [-1], [0, 1]
    for w in widths:
        parents += [p for p in range(levels[-2], levels[-1]) for _ in range(w)]
        levels.append(len(parents))
    return parents, levels


class Drafting:
    """Rounds of drafts and verdicts over texts (lists of token ids, one a sequence)."""

    def __init__(self, small, large, texts, widths, temperature, seed=0):
        self.small, self.large, self.texts = small, large, [list(t) for t in texts]
        self.parents, self.levels = parents_of(widths)
        self.temperature, self.rows = temperature, len(self.parents)
        n = len(texts)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.verifier = B.DraftVerifier(large.cfg["vocab"], n * self.rows, max_width=max([1, *widths]))
        self.widths, self.trees = widths, {}                  # trees: of the first levels, by their rows
        small.read(self.texts, [len(t) - 1 for t in texts])
        large.read(self.texts, [len(t) - 1 for t in texts])

    def _spans(self, model, rows):
        spans = [(s, n, n, rows) for s, n in enumerate(model.len)]
        if rows not in self.trees:
            self.trees[rows] = B.DraftSpans(spans, [self.parents[:rows]] * len(self.texts))
        return self.trees[rows].at(spans)

    def draft(self):
        """Tokens of the trees [sequences][rows], and the small model's logits after every row but the last level's (zeros there)."""
        n, vocab = len(self.texts), self.small.cfg["vocab"]
        tokens = torch.zeros(n, self.rows, dtype=torch.int32, device="cuda")
        tokens[:, 0] = torch.tensor([t[-1] for t in self.texts], device="cuda")
        logits = torch.zeros(n, self.rows, vocab, device="cuda")
        for level, w in enumerate(self.widths):
            lo, hi = self.levels[level], self.levels[level + 1]
            got = self.small.forward(tokens[:, :hi].flatten(), self._spans(self.small, hi)).view(n, hi, vocab)[:, lo:hi]
            logits[:, lo:hi] = got
            if self.temperature > 0:                          # each drawn by itself
                new = torch.multinomial(torch.softmax(got.flatten(0, 1) / self.temperature, -1), w, replacement=True, generator=self.gen)
            else:
                new = got.flatten(0, 1).topk(w).indices
            tokens[:, hi:hi + w * (hi - lo)] = new.view(n, -1).int()
        return tokens, logits

    def round(self):
        """One round; returns how many tokens each text has grown by."""
        n = len(self.texts)
        tokens, drafted = self.draft()
        spans = self._spans(self.large, self.rows)
        target = self.large.forward(tokens.flatten(), spans)
        accept = torch.rand(n * self.rows, dtype=torch.float64, device="cuda", generator=self.gen)
        sample = torch.rand(n, dtype=torch.float64, device="cuda", generator=self.gen)
        path, accepted, after = self.verifier.verify(spans, tokens.flatten(), target, self.temperature, accept, sample, draft=drafted.flatten(0, 1) if self.temperature > 0 else None)
        counts, steps, last, written = accepted.tolist(), path.tolist(), after.tolist(), tokens.tolist()
        self.large.keep(spans, path, accepted, counts)
        for s in range(n):
            self.texts[s] += [written[s][r] for r in steps[s][:counts[s]]] + [last[s]]
        self.small.read(self.texts, [len(t) - 1 for t in self.texts])     # (what it wrote on other branches is written over)
        return [c + 1 for c in counts]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--small", default="qwen7b", choices=synth.SHAPES)
    ap.add_argument("--large", default="qwen32b", choices=synth.SHAPES)
    ap.add_argument("--layers", type=int, default=4, help="layers of each model (0: all)")
    ap.add_argument("--sequences", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=256)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--widths", type=int, nargs="+", default=[1, 1, 1, 1])
    ap.add_argument("--temperature", type=float, default=0.6)
    a = ap.parse_args(argv)
    rows = len(parents_of(a.widths)[0])
    longest = a.prompt + a.tokens + 2 * rows + 8
    small, large = (PagedModel(m, i, a.sequences, longest, max(rows, 64), a.layers or None) for i, m in enumerate((a.small, a.large)))
    vocab = min(small.cfg["vocab"], large.cfg["vocab"])
    if small.cfg["vocab"] != large.cfg["vocab"]:
        raise SystemExit("the models have different vocabularies")
    prompts = [synth.make_prompt(a.prompt, vocab, 7 + s).tolist() for s in range(a.sequences)]
    job = Drafting(small, large, prompts, a.widths, a.temperature)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    rounds = grown = 0
    start.record()
    while max(len(t) for t in job.texts) < a.prompt + a.tokens:
        grown += sum(job.round())
        rounds += 1
    end.record()
    end.synchronize()
    print(f"{a.sequences} sequences, prompt of {a.prompt}, trees of {rows} rows: {rounds} rounds, {grown / (rounds * a.sequences):.2f} tokens a round and sequence, "
          f"{start.elapsed_time(end) / rounds:.2f} ms a round")


if __name__ == "__main__":
    main()
