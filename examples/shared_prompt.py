"""One attention layer that serves many sequences behind one prompt, and a step that trains what prepares its queries and keys.

    python examples/shared_prompt.py [--prompt 32768] [--batch 16] [--question 200] [--steps 32]

The prompt is fed once, into a cache of its own.  Every sequence then asks a question (many tokens: attention over itself,
joined with that over the prompt) and is decoded token by token (both in one call).  In each, one launch turns the
projection's rows into normed, rotated queries and keys and values in the layout that the cache's calls take.
Weights and hidden states are random."""

from __future__ import annotations

import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2605_14037_amd as spkv  # noqa: E402


class Layer:
    """Projection, norms of the heads, rotation and utility predictor of one layer."""

    def __init__(self, d_model=1024, q_heads=32, kv_heads=8, head_dim=128, theta=1e6, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.q_heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        self.rope = spkv.Rope(head_dim, theta=theta)

        def randn(*shape):
            return torch.randn(*shape, generator=g, device="cuda")

        self.qkv = (randn((q_heads + 2 * kv_heads) * head_dim, d_model) / d_model ** 0.5).bfloat16()
        self.norm = {"q_weight": 1 + 0.1 * randn(head_dim), "k_weight": 1 + 0.1 * randn(head_dim), "eps": 1e-6}
        hidden = 256
        self.predictor = ((randn(hidden, d_model) / d_model ** 0.5).bfloat16(), 0.1 * randn(hidden),
                          (4.0 * randn(kv_heads, hidden) / hidden ** 0.5).bfloat16(), randn(kv_heads) - 0.5)

    def rows(self, hidden):
        """The projection's rows, and the heads of queries, keys and values in them (no copies)."""
        rows = (hidden @ self.qkv.t()).view(len(hidden), -1, self.head_dim)
        return rows, rows.split([self.q_heads, self.kv_heads, self.kv_heads], 1)

    def prepare(self, hidden, positions):
        """Queries, keys, values and utility logits of tokens at their positions."""
        q, k, v = self.rows(hidden)[1]
        return spkv.qk_norm_rope(q, k, positions, self.rope, v=v, **self.norm) + (spkv.utility_logits(hidden, *self.predictor),)

    def cache(self, sequences, tokens):
        return spkv.SPKVCache(sequences, self.q_heads, self.kv_heads, self.head_dim, max_context=tokens,
                              max_total_kept_tokens=sequences * self.kv_heads * tokens)


def serve(layer, prompt, questions, answers):
    """prompt [P, d_model]; questions: a list of [n, d_model]; answers: [steps, batch, d_model].  Returns the attention of
    the questions' tokens [sum n, H_q, D] and of every step [steps, batch, H_q, D]."""
    batch, steps, start = len(questions), len(answers), len(prompt)
    place = torch.arange(start, device="cuda", dtype=torch.int32)
    prompts = layer.cache(1, start)
    for at in range(0, start, 4096):
        _, k, v, f = layer.prepare(prompt[at:at + 4096], place[at:at + 4096])
        prompts.append(k, v, f, [0, len(k)])

    lengths = [len(x) for x in questions]
    cu = [sum(lengths[:b]) for b in range(batch + 1)]
    cache = layer.cache(batch, max(lengths) + steps)
    sharing = spkv.PrefixSharing(prompts, [0] * batch)
    positions = torch.cat([torch.arange(start, start + n, device="cuda", dtype=torch.int32) for n in lengths])
    q, k, v, f = layer.prepare(torch.cat(questions), positions)
    own, lse = cache.prefill_attention(k, v, f, q, cu, want_lse=True)
    asked, _ = cache.prefix_attention(sharing, q, cu, own, lse, out=own, lse=lse)

    positions = torch.tensor([start + n for n in lengths], device="cuda", dtype=torch.int32)
    workspace = torch.empty(sharing.workspace_bytes(batch), dtype=torch.uint8, device="cuda")
    one_each = cache.make_cu(range(batch + 1))
    out = torch.empty(steps, batch, layer.q_heads, layer.head_dim, dtype=torch.bfloat16, device="cuda")
    for step in range(steps):
        q, k, v, f = layer.prepare(answers[step], positions)
        cache.append(k, v, f, one_each)
        cache.decode_attention_shared(sharing, q, out=out[step], workspace=workspace)
        positions += 1
    return asked, out


def whole(layer, prompt, question, answers):
    """The same for one sequence that holds the prompt itself: attention of the question's tokens and of every step."""
    hidden = torch.cat([prompt, question])
    cache = layer.cache(1, len(hidden) + len(answers))
    place = torch.arange(len(hidden) + len(answers), device="cuda", dtype=torch.int32)
    asked, out = [], []
    for at, end in [(i, min(i + 4096, len(prompt))) for i in range(0, len(prompt), 4096)] + [(len(prompt), len(hidden))]:
        q, k, v, f = layer.prepare(hidden[at:end], place[at:end])
        asked = cache.prefill_attention(k, v, f, q, [0, end - at])
    for step in range(len(answers)):
        q, k, v, f = layer.prepare(answers[step:step + 1], place[len(hidden) + step:len(hidden) + step + 1])
        out.append(cache.decode_step(k, v, f, q))
    return asked, torch.cat(out)


def train_step(layer, hidden, positions, wanted, rate):
    """One step of gradient descent on the projection and the norms' weights towards `wanted` queries, keys and values (of
    a teacher).  Returns the loss before it, half the mean squared distance."""
    rows, (q, k, v) = layer.rows(hidden)
    got = spkv.qk_norm_rope(q, k, positions, layer.rope, v=v, **layer.norm)
    off = [a.float() - b.float() for a, b in zip(got, wanted)]
    count = sum(x.numel() for x in off)
    dq, dk, dv = [(x * (rate / count)).bfloat16() for x in off]
    grad = torch.empty_like(rows)
    parts = grad.split([layer.q_heads, layer.kv_heads, layer.kv_heads], 1)
    dq_weight, dk_weight = spkv.qk_norm_rope_backward(dq, dk, positions, layer.rope, q=q, k=k, dv=dv, out=parts, **layer.norm)
    layer.qkv = (layer.qkv.float() - (grad.view(len(hidden), -1).t() @ hidden).float()).bfloat16()
    layer.norm["q_weight"] -= dq_weight
    layer.norm["k_weight"] -= dk_weight
    return 0.5 * sum(x.square().sum() for x in off).item() / count


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--prompt", type=int, default=32768)
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--question", type=int, default=200, help="tokens of the longest question")
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--d-model", type=int, default=1024)
    ap.add_argument("--heads", type=int, nargs=3, default=(32, 8, 128), metavar=("H_q", "H_kv", "D"))
    a = ap.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(1)

    def hidden(*shape):
        return torch.randn(*shape, a.d_model, generator=g, device="cuda").bfloat16()

    layer = Layer(a.d_model, *a.heads)
    prompt, answers = hidden(a.prompt), hidden(a.steps, a.batch)
    questions = [hidden(1 + b * (a.question - 1) // max(a.batch - 1, 1)) for b in range(a.batch)]
    serve(layer, prompt, questions, answers[:1])
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    asked, out = serve(layer, prompt, questions, answers)
    torch.cuda.synchronize()
    took = time.perf_counter() - t0
    last_asked, last_out = whole(layer, prompt, questions[-1], answers[:, -1])

    def apart(x, y):
        return ((x.float() - y.float()).norm() / y.float().norm()).item()

    report = {"ms": 1e3 * took, "apart_question": apart(asked[-len(questions[-1]):], last_asked), "apart_steps": apart(out[:, -1], last_out)}
    print(f"{a.batch} sequences behind a prompt of {a.prompt} tokens: prompt, questions and {a.steps} steps {report['ms']:.1f} ms; "
          f"the last sequence alone differs by {report['apart_question']:.1e} (question), {report['apart_steps']:.1e} (steps)")

    student = Layer(a.d_model, *a.heads, seed=0)
    student.norm["q_weight"], student.norm["k_weight"] = torch.ones(2, a.heads[2], device="cuda").unbind(0)
    x, place = hidden(512), torch.arange(512, device="cuda", dtype=torch.int32)
    wanted = layer.prepare(x, place)[:3]
    # (the loss curves by at most about H_q / ((H_q + 2 H_kv) D) along a weight of the norms: steps well below its inverse)
    report["losses"] = [train_step(student, x, place, wanted, rate=0.5 * a.heads[2]) for _ in range(5)]
    print("losses of five steps towards the layer's norms:", " ".join(f"{v:.2e}" for v in report["losses"]))
    return report


if __name__ == "__main__":
    main()
