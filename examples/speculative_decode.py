"""Speculative decoding with one multi-scale model: the narrow bitwidth drafts, the wide one verifies.

A small random Llama-shaped model whose every linear is served by the library.  Per step the draft proposes a chain of tokens, one GEMV a
linear at DRAFT bits each; the target then runs all of them and the token before at once, a batch of up to 8 right-hand sides at TARGET bits:
rotary positions, attention of the drafted tokens over the paged cache and over one another, verification, and the keys and values of
the tokens that stand go into the cache.  The norms, the activation and the embedding are torch.

    python examples/speculative_decode.py            # prints how many tokens a step yields, and the speed beside plain decoding
"""
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2508_06041_amd as dp  # noqa: E402
import synth  # noqa: E402

BLOCKS, WIDTH, HEADS, KV, DIM, INNER, WORDS = 2, 512, 8, 4, 64, 1024, 1000
DRAFT, TARGET, NODES, PAGE = 4, 8, 6, 16
Q, K, V, O, GATE, UP, DOWN = range(7)


class Decoder:
    def __init__(self, seed=0, pages=32):
        shapes = [(HEADS * DIM, WIDTH), (KV * DIM, WIDTH), (KV * DIM, WIDTH), (WIDTH, HEADS * DIM), (INNER, WIDTH), (INNER, WIDTH), (WIDTH, INNER)]
        self.model = dp.Model(BLOCKS * 7 + 1)
        for i, (out, in_) in enumerate(shapes * BLOCKS + [(WORDS, WIDTH)]):
            lin = synth.make_linear(out, in_, TARGET, DRAFT, seed=1000 * seed + i)
            size = lin["luts"][TARGET].float().square().mean().sqrt().item() * in_ ** 0.5
            self.model.dpllm_load_linear(i, synth.planes_np(lin["planes"]), {k: synth.lut_np((t.float() / size).half()) for k, t in lin["luts"].items()}, DRAFT)
        g = torch.Generator().manual_seed(seed)
        self.embedding = torch.randn(WORDS, WIDTH, generator=g).half().cuda()
        self.uniforms = torch.Generator(device="cuda").manual_seed(seed)
        self.freqs, self.scale = dp.dpllm_rope_frequencies(DIM, 10000.0, dp.DPLLM_ROPE_BANDS, 8.0, 1024, 1.0, 4.0)
        self.k, self.v = (torch.zeros(BLOCKS, pages, PAGE, KV, DIM, dtype=torch.float16, device="cuda") for _ in range(2))
        table = torch.randperm(pages, generator=g).to(torch.int32)[None].cuda()
        self.cache = dp.Cache(self.k, self.v, table)
        self.lens = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.new_k, self.new_v = (torch.zeros(BLOCKS, 1, NODES, KV, DIM, dtype=torch.float16, device="cuda") for _ in range(2))
        self.queries = torch.zeros(BLOCKS, 1, NODES, HEADS, DIM, dtype=torch.float16, device="cuda")

    def forward(self, tokens, first, bits):
        """Logits [n][words] behind nodes first ... of the chain; their keys and values go to new_k, new_v, over the nodes before them."""
        n, end = tokens.shape[0], first + tokens.shape[0]
        x = self.embedding[tokens.long()].float()
        positions = (self.lens + torch.arange(first, end, device="cuda")).to(torch.int32)

        def norm(y):
            return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-5)).half()
        for b in range(BLOCKS):
            def linear(i, y):
                return self.model.dpllm_gemv(7 * b + i, bits, y.contiguous())
            h = norm(x)
            heads = [linear(i, h).view(1, n, -1, DIM) for i in (Q, K, V)]
            dp.dpllm_rope((heads[0], heads[1]), positions, self.freqs, out=(self.queries[b][:, first:end], self.new_k[b][:, first:end]), scale=self.scale)
            self.new_v[b][:, first:end] = heads[2]
            # a chain: every node sees the context, the nodes before it and itself
            y = dp.dpllm_tree_attention(self.cache, b, self.lens, self.queries[b][:, :end], self.new_k[b][:, :end], self.new_v[b][:, :end])
            x = x + linear(O, y[0, first:].reshape(n, -1)).float()
            h = norm(x)
            x = x + linear(DOWN, (torch.nn.functional.silu(linear(GATE, h).float()) * linear(UP, h).float()).half()).float()
        return self.model.dpllm_gemv(BLOCKS * 7, bits, norm(x))

    def step(self, token, temperature, nodes):
        """One step behind `token`, int32 [1]: the tokens it yields, int32 [nodes] with -1 behind them, and how many."""
        tokens = torch.zeros(1, nodes, dtype=torch.int32, device="cuda")
        tokens[0, :1] = token
        draft = torch.zeros(1, nodes, WORDS, dtype=torch.float16, device="cuda")
        t = max(temperature, 0.01)
        for i in range(nodes - 1):
            draft[0, i] = self.forward(tokens[0, i:i + 1], i, DRAFT)[0]
            p = torch.softmax(draft[0, i].float() / t, 0)
            tokens[0, i + 1] = p.argmax() if temperature == 0 else torch.multinomial(p, 1, generator=self.uniforms)[0]
        logits = self.forward(tokens[0], 0, TARGET)
        uniforms = torch.rand(1, nodes, device="cuda", generator=self.uniforms)
        count, path, words = dp.dpllm_verify(logits[None], tokens, uniforms, torch.full((1,), temperature, device="cuda"), draft=draft)
        dp.dpllm_cache_append(self.cache, self.lens, self.new_k[:, :, :nodes], self.new_v[:, :, :nodes], path=path, count=count)
        self.lens += count
        return words[0], count

    def decode(self, token, n, temperature=0.0, nodes=NODES):
        """At least n tokens behind `token`, as a list, and the number of steps."""
        out, steps = [], 0
        last = torch.tensor([token], dtype=torch.int32, device="cuda")
        while len(out) < n:
            words, count = self.step(last, temperature, nodes)
            c = count.item()
            out += words[:c].tolist()
            last = words[c - 1:c]
            steps += 1
        return out, steps


def main():
    for temperature in (0.0, 0.7):
        for nodes in (1, NODES):
            d = Decoder()
            d.decode(1, 2, temperature, nodes)
            torch.cuda.synchronize()
            start = time.time()
            out, steps = d.decode(1, 100, temperature, nodes)
            print("temperature %.1f, %d drafted: %.2f tokens a step, %.0f tokens/s" % (temperature, nodes - 1, len(out) / steps, len(out) / (time.time() - start)))
            d.model.close()


if __name__ == "__main__":
    main()
