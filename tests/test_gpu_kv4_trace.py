"""The trace over two 4-bit caches, every call of its models checked: appended slots against the quantised rows, attention against the slots' values
in 64 bits, evictions against the ledger's order (kv4_ref; tolerances of test_gpu_kv4)."""
import numpy as np
import pytest
import torch

from paper_2504_12329_amd import binding as B
from paper_2504_12329_amd import kv4_trace

from . import kv4_ref as R
from .test_gpu_kv4 import WEIGHT_TOL, f64, out_tol

pytestmark = pytest.mark.gpu


class Checked:
    """A cache whose calls are followed by a plain one: its slots per layer and sequence, [nkv][slots][d] in 64 bits."""

    def __init__(self, kv):
        self.kv, self.held, self.calls = kv, {}, {"append": 0, "attend": 0, "evict": 0}

    def append(self, layer, spans, qkv, q_norm=None, k_norm=None, ledger=None):
        q = self.kv.append(layer, spans, qkv, q_norm, k_norm, ledger)
        k, v = (f64(t[0]) for t in self.kv.read(layer, layer + 1, spans))
        c, at = self.kv.cfg, 0
        values = f64(qkv).reshape(-1, c["n_q_heads"] + 2 * c["n_kv_heads"], c["head_dim"])[:, c["n_q_heads"] + c["n_kv_heads"]:]
        for seq, n, pos, r in spans.spans:
            if r:
                codes, scales = R.quantise(values[at:at + r])
                assert np.array_equal(v[at:at + r], R.values(codes, scales))
                held = self.held.get((layer, seq), (np.zeros((c["n_kv_heads"], 0, c["head_dim"])),) * 2)
                self.held[layer, seq] = tuple(np.concatenate([a[:, :n], b[at:at + r].transpose(1, 0, 2)], 1) for a, b in zip(held, (k, v)))
                assert (ledger.positions[layer, seq, :, n:n + r].cpu().numpy() == np.arange(pos, pos + r)).all()
            at += r
        self.calls["append"] += 1
        return q

    def attend(self, layer, spans, q, ledger):
        c, at = self.kv.cfg, 0
        before = f64(ledger.weights[layer])
        out = self.kv.attend(layer, spans, q, ledger)
        got, qs = f64(out), f64(q)
        for seq, n, _, r in spans.spans:
            want, size, w = R.attention(qs[at:at + r], *self.held[layer, seq], n)
            assert (np.abs(got[at:at + r] - want) <= out_tol(want, size)).all(), (layer, seq, n, r)
            before[seq, :, :n + r] += w
            at += r
        assert (np.abs(f64(ledger.weights[layer]) - before) <= WEIGHT_TOL * before).all()
        self.calls["attend"] += 1
        return out

    def evict(self, lo, hi, spans, keep, recent, ledger):
        w, p = ledger.weights.cpu().numpy(), ledger.positions.cpu().numpy()
        self.kv.evict(lo, hi, spans, keep, recent, ledger)
        now_w, now_p = ledger.weights.cpu().numpy(), ledger.positions.cpu().numpy()
        for seq, n, pos, _ in spans.spans:
            k, v = (f64(t) for t in self.kv.read(lo, hi, B.Kv4Spans([(seq, 0, 0, keep)])))
            for layer in range(lo, hi):
                held = self.held[layer, seq]
                src = [R.evict(w[layer, seq, h, :n], p[layer, seq, h, :n], pos, keep, recent) for h in range(len(held[0]))]
                held = self.held[layer, seq] = tuple(np.stack([a[h, s] for h, s in enumerate(src)]) for a in held)
                for h, s in enumerate(src):
                    assert np.array_equal(now_w[layer, seq, h, :keep], w[layer, seq, h, s])
                    assert np.array_equal(now_p[layer, seq, h, :keep], p[layer, seq, h, s])
                for a, b in zip(held, (k, v)):
                    assert np.array_equal(a, b[layer - lo].transpose(1, 0, 2))
        self.calls["evict"] += 1


def test_a_trace_call_by_call():
    print("trace over two caches", flush=True)
    models = [kv4_trace.Context(name, 1, n_seq=2, max_pos=200, budget=48, recent=8, max_rows=24) for name in ("tiny_small", "tiny_large")]
    for m in models:
        m.kv = Checked(m.kv)
    wrote, out = kv4_trace.trace(*models, 2, prompt=40, tokens=70, segment=20, takeover=7)
    assert wrote == {"small": 56, "large": 14}
    for m, name in zip(models, ("small", "large")):
        assert m.slots[0] <= 72 and m.evictions == m.kv.calls["evict"] >= 2
        assert torch.isfinite(out[name]).all()
        assert m.kv.calls["append"] == m.kv.calls["attend"] > 0
    assert models[0].pos == [110, 110] and models[1].pos == [94, 94]        # (the large one has not read the last 16 tokens)


def test_the_command(capsys):
    print("the command", flush=True)
    kv4_trace.main(["--small", "tiny_small", "--large", "tiny_large", "--layers", "0", "--sequences", "3", "--prompt", "70", "--tokens", "200",
                    "--budget", "96", "--recent", "16", "--rows", "64"])
    said = capsys.readouterr().out
    assert "3 sequences, prompt of 70" in said and "after 2 evictions" in said
