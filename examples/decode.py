"""A decoder answers several prompts beside a vision tenant on one GPU.

The decoder (random weights) is written down as operator lists (paper_2304_11745_amd.tokens): one that takes whole prompts, one
that takes a token of every sequence, and the head that turns hidden states into the next tokens.  Prompts are filled in and
decoded with gacer_enqueue, step after step without waiting; then a decoding step and a ResNet-18 run in the same rounds, unsplit and with the
batch of every operator cut in two.

    python examples/decode.py [--steps 32] [--batch 6] [--dtype bf16] [--weights fp8]

With --weights fp8 the projections and the feed-forward block hold 8-bit weights and read 8-bit rows: RMS norms with the residual's addition leave the rows, a
gated block takes the place of the two products around an activation.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2304_11745_amd import binding as B  # noqa: E402
from paper_2304_11745_amd import harness, tokens as T  # noqa: E402


class Decoder:
    """Two lists over shared weights and caches: a pre-norm decoder of `layers` layers with `heads` query and `kv` key/value heads."""

    def __init__(self, dtype=torch.bfloat16, batch=6, layers=2, heads=8, kv=2, dim=64, ffn=1024, vocab=8000, longest=160, page=32, seed=1, fp8=False):
        self.fp8 = fp8
        self.dtype, self.batch, self.layers, self.heads, self.kv, self.dim, self.ffn, self.vocab = dtype, batch, layers, heads, kv, dim, ffn, vocab
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        width = self.width = heads * dim
        self.embedding = self.normal(vocab, width)
        self.layer = [dict(n1=self.norm(), n2=self.norm(), qkv=self.normal((heads + 2 * kv) * dim, width, scale=width ** -0.5), gq=torch.ones(dim, device="cuda"),
                           gk=torch.ones(dim, device="cuda"), o=self.normal(width, width, scale=width ** -0.5), up=self.normal(ffn, width, scale=width ** -0.5),
                           down=self.normal(width, ffn, scale=ffn ** -0.5)) for _ in range(layers)]
        if fp8:
            for p in self.layer:
                p["gate"] = self.normal(ffn, width, scale=width ** -0.5)
                for name in ("qkv", "o", "gate", "up", "down"):
                    p[name] = T.Fp8Weight.quantise(p[name])
        self.last, self.out = self.norm(), self.normal(vocab, width, scale=3 * width ** -0.5)
        angle = torch.arange(longest, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(dim // 2, device="cuda", dtype=torch.float64) * 2 / dim)
        self.table = torch.stack((angle.cos(), angle.sin()), -1).float().contiguous()
        per = -(-longest // page)
        pages = torch.randperm(batch * per, generator=self.gen, device="cuda").to(torch.int32).reshape(batch, per)
        self.caches = [T.Cache.allocate(batch * per, kv, dim, pages, page) for _ in range(layers)]
        self.start = torch.zeros(batch, dtype=torch.int32, device="cuda")

    def normal(self, *shape, scale=1.0):
        return (scale * torch.randn(shape, generator=self.gen, device="cuda")).to(self.dtype)

    def norm(self):
        return torch.ones(self.width, device="cuda"), torch.zeros(self.width, device="cuda")

    def empty(self, tokens, features):
        return torch.empty(self.batch, tokens, features, dtype=self.dtype, device="cuda")

    def body(self, tokens, count=None):
        """The list that takes `tokens` new tokens of every sequence: (list, its input, its positions, its hidden states)."""
        ops = T.OpList(self.dtype, self.batch)
        x = first = self.empty(tokens, self.width)
        positions = torch.zeros(self.batch, tokens, 1, dtype=torch.int32, device="cuda")
        heads = dict(heads=self.heads, kv_heads=self.kv, head_dim=self.dim)
        if self.fp8:
            return ops, first, positions, self.body_fp8(ops, x, tokens, count, positions, heads)
        for p, cache in zip(self.layer, self.caches):
            h, qkv, ctx, y = self.empty(tokens, self.width), self.empty(tokens, (self.heads + 2 * self.kv) * self.dim), self.empty(tokens, self.width), self.empty(tokens, self.width)
            ops.layernorm(x, *p["n1"], h)
            ops.gemm(h, p["qkv"], qkv)
            ops.qknorm_rope(qkv, qkv, positions, self.table, gamma_q=p["gq"], gamma_k=p["gk"], **heads)
            ops.cache_write(qkv, cache, self.start, count, **heads)
            ops.cache_attention(qkv, ctx, cache, self.start, count, **heads)
            ops.gemm(ctx, p["o"], y, res=x)
            h2, f, z = self.empty(tokens, self.width), self.empty(tokens, self.ffn), self.empty(tokens, self.width)
            ops.layernorm(y, *p["n2"], h2)
            ops.gemm(h2, p["up"], f, act="gelu")
            ops.gemm(f, p["down"], z, res=y)
            x = z
        return ops, first, positions, x

    def body_fp8(self, ops, x, tokens, count, positions, heads):
        """The layers with 8-bit rows and weights: every product reads the rows that the operator before it left."""
        for p, cache in zip(self.layer, self.caches):
            rows, qkv, ctx = T.Fp8Rows.allocate(self.batch, tokens, self.width), self.empty(tokens, (self.heads + 2 * self.kv) * self.dim), self.empty(tokens, self.width)
            ops.rmsnorm_fp8(x, rows, p["n1"][0])
            ops.gemm_fp8(rows, p["qkv"], qkv)
            ops.qknorm_rope(qkv, qkv, positions, self.table, gamma_q=p["gq"], gamma_k=p["gk"], **heads)
            ops.cache_write(qkv, cache, self.start, count, **heads)
            ops.cache_attention(qkv, ctx, cache, self.start, count, **heads)
            rows, y = T.Fp8Rows.allocate(self.batch, tokens, self.width), self.empty(tokens, self.width)
            ops.quantise_fp8(ctx, rows)
            ops.gemm_fp8(rows, p["o"], y)
            rows, inner, h, z = T.Fp8Rows.allocate(self.batch, tokens, self.width), T.Fp8Rows.allocate(self.batch, tokens, self.ffn), self.empty(tokens, self.width), self.empty(tokens, self.width)
            ops.rmsnorm_fp8(y, rows, p["n2"][0], res=x, sum=h)
            ops.gated_fp8(rows, p["gate"], p["up"], inner)
            ops.gemm_fp8(inner, p["down"], z, res=h)
            x = z
        return x

    def head(self, ops, x, token, u, **filters):
        """Final norm, logits and sampling of hidden states [batch, 1, width] at the end of a list."""
        h, logits = self.empty(1, self.width), self.empty(1, self.vocab)
        if self.fp8:
            ops.rmsnorm(x, self.last[0], h)
        else:
            ops.layernorm(x, *self.last, h)
        ops.gemm(h, self.out, logits)
        ops.sample(logits, token, u, **filters)
        return logits


def serve(dtype=torch.bfloat16, batch=6, steps=32, vision=True, seed=1, **sizes):
    """Fills prompts in and decodes; returns (tokens [batch, steps + 1], logits of the last step)."""
    d = Decoder(dtype, batch, seed=seed, **sizes)
    longest = 40
    lengths = torch.tensor([1 + (7 * i) % longest for i in range(batch)], dtype=torch.int32, device="cuda")
    prompts = torch.randint(0, d.vocab, (batch, longest), generator=d.gen, device="cuda")
    token, u = torch.zeros(batch, dtype=torch.int32, device="cuda"), torch.empty(batch, device="cuda")
    filters = dict(temperature=torch.full((batch,), 0.8, device="cuda"), top_k=torch.full((batch,), 50, dtype=torch.int32, device="cuda"),
                   top_p=torch.full((batch,), 0.95, device="cuda"))

    fill, fill_in, fill_at, fill_out = d.body(longest, lengths)
    first_head, tail = T.OpList(dtype, batch), d.empty(1, d.width)
    d.head(first_head, tail, token, u, **filters)
    step, step_in, step_at, step_out = d.body(1)
    logits = d.head(step, step_out, token, u, **filters)
    session = T.TokenSession([fill, first_head, step])

    # prompts: all tokens at once, the last real one of each sequence goes to the head
    fill_in.copy_(d.embedding[prompts])
    fill_at.copy_(torch.arange(longest, device="cuda", dtype=torch.int32)[None, :, None].expand_as(fill_at))
    session.enqueue(0)
    tail.copy_(fill_out[torch.arange(batch, device="cuda"), lengths.long() - 1][:, None])
    u.copy_(torch.rand(batch, generator=d.gen, device="cuda"))
    session.enqueue(1)
    d.start.copy_(lengths)
    said = [token.clone()]
    torch.cuda.synchronize()
    begin = time.perf_counter()
    for _ in range(steps):
        step_in.copy_(d.embedding[token.long()][:, None])
        step_at.copy_(d.start[:, None, None])
        u.copy_(torch.rand(batch, generator=d.gen, device="cuda"))
        session.enqueue(2)
        d.start.add_(1)
        said.append(token.clone())
    torch.cuda.synchronize()
    print("%d sequences, %d steps: %.0f us a step" % (batch, steps, (time.perf_counter() - begin) / max(1, steps) * 1e6))
    result = torch.stack(said, 1), logits.clone()
    if vision:
        import synth
        tenants, data = synth.build_config(2)
        rounds = harness.Session(tenants[:1], data[:1], extra=[step])
        for name, splits in (("unsplit", []), ("batch in two", rounds.uniform_splits("batch", 2))):
            rounds.set_plan(splits, [])
            rounds.run(B.GACER_MODE_PLAN, 3)
            ms = sorted(rounds.run(B.GACER_MODE_PLAN, 20))[10]
            print("a step beside %s (%d images): %.0f us a round, %s" % (tenants[0].name, tenants[0].batch, ms * 1e3, name))
        rounds.close()
    session.close()
    return result


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--batch", type=int, default=6)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    ap.add_argument("--weights", choices=("full", "fp8"), default="full")
    a = ap.parse_args()
    said, _ = serve(torch.bfloat16 if a.dtype == "bf16" else torch.float32, a.batch, a.steps, fp8=a.weights == "fp8")
    for row in said.tolist():
        print(" ".join(map(str, row[:12])), "..." if len(row) > 12 else "")
