"""Decoding over a cache of keys and values in 8 or 4 bits.

The model of speculative_decode.py with learned norms of the heads of queries and keys.  Per step: norms and rotary positions in one call, attention of the new tokens over the quantised cache and over one
another, the new keys and values quantised into the cache, and a draw with temperature, top-k, top-p and min-p.

    python examples/quantized_decode.py            # prints bytes of cache a token, how far attention is from that over 16 bits, and the speed, format by format
"""
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import speculative_decode as plain  # noqa: E402

from speculative_decode import BLOCKS, DIM, DOWN, GATE, HEADS, K, KV, O, PAGE, Q, TARGET, UP, V, WORDS, dp  # noqa: E402

FORMATS = {"e4m3": dp.DPLLM_CACHE_E4M3, "int8": dp.DPLLM_CACHE_INT8, "int4": dp.DPLLM_CACHE_INT4}
ROWS = 8      # tokens of a prompt at once: what a GEMV takes


class Decoder(plain.Decoder):
    def __init__(self, form, seed=0, pages=32):
        super().__init__(seed, pages)
        self.cache = dp.QuantizedCache.zeros(FORMATS[form], BLOCKS, pages, PAGE, KV, DIM, self.cache.table)
        g = torch.Generator().manual_seed(seed + 1)
        self.norms = [tuple((1 + 0.1 * torch.randn(DIM, generator=g)).cuda() for _ in range(2)) for _ in range(BLOCKS)]
        self.draws = torch.Generator(device="cuda").manual_seed(seed + 2)

    def forward(self, tokens):
        """Logits [n][words] behind the n tokens, which come behind those in the cache and go into it."""
        n = tokens.shape[0]
        x = self.embedding[tokens.long()].float()
        positions = (self.lens + torch.arange(n, device="cuda")).to(torch.int32)

        def norm(y):
            return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-5)).half()
        new_k, new_v = (torch.empty(BLOCKS, 1, n, KV, DIM, dtype=torch.float16, device="cuda") for _ in range(2))
        for b in range(BLOCKS):
            def linear(i, y):
                return self.model.dpllm_gemv(7 * b + i, TARGET, y.contiguous())
            h = norm(x)
            q, k, v = [linear(i, h).view(1, n, -1, DIM) for i in (Q, K, V)]
            new_v[b] = v
            dp.dpllm_norm_rope((q, k), self.norms[b], positions, self.freqs, scale=self.scale, out=(q, new_k[b]))
            self.last = b, q, new_k[b], new_v[b], dp.dpllm_quantized_attention(self.cache, b, self.lens, q, new_k[b], new_v[b])
            x = x + linear(O, self.last[-1].view(n, -1)).float()
            h = norm(x)
            x = x + linear(DOWN, (torch.nn.functional.silu(linear(GATE, h).float()) * linear(UP, h).float()).half()).float()
        dp.dpllm_quantized_append(self.cache, self.lens, new_k, new_v)
        self.lens += n
        return self.model.dpllm_gemv(BLOCKS * 7, TARGET, norm(x))

    def decode(self, prompt, n, temperature=0.0, top_k=None, top_p=None, min_p=None):
        """n words behind the prompt, and how many could have been drawn in place of each."""
        def one(v, dtype=torch.float32):
            return None if v is None else torch.tensor([v], dtype=dtype, device="cuda")
        how = dict(temperature=one(temperature), top_k=one(top_k, torch.int32), top_p=one(top_p), min_p=one(min_p))
        tokens = torch.tensor(prompt, dtype=torch.int32, device="cuda")
        words, kept = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
        uniforms = torch.rand(n, generator=self.draws, device="cuda")
        for first in range(0, len(prompt), ROWS):
            logits = self.forward(tokens[first:first + ROWS])
        for i in range(n):
            dp.dpllm_sample(logits[-1:], uniforms[i:i + 1], words=words[i:i + 1], kept=kept[i:i + 1], **how)
            if i + 1 < n:
                logits = self.forward(words[i:i + 1])
        return words.tolist(), kept.tolist()

    def in_16_bits(self):
        """What the cache holds, as a Cache in 16 bits of one page."""
        n = self.lens.item()
        k, v = dp.dpllm_quantized_read(self.cache, None, n, torch.float16, layers=BLOCKS)
        return dp.Cache(k, v)


def main():
    for form in FORMATS:
        d = Decoder(form)
        d.decode([1, 2, 3], 2)
        torch.cuda.synchronize()
        start = time.time()
        words, kept = d.decode(list(range(20)), 200, 0.8, top_k=50, top_p=0.95, min_p=0.02)
        seconds = time.time() - start
        b, q, k, v, got = d.last
        wide = d.in_16_bits()
        before = d.lens - 1      # the last token came behind these
        want = dp.dpllm_tree_attention(wide, b, before, q, k, v)
        size = sum(t[0, 0, 0].numel() * t.element_size() for t in (d.cache.k, d.cache.v, d.cache.k_scales, d.cache.v_scales))
        print("%s: %d bytes a token and layer (%d in 16 bits), attention %.1e off, %.0f words of %d to draw from, %.0f tokens/s" % (
            form, size, 4 * KV * DIM, (got.float() - want.float()).norm() / want.float().norm(), sum(kept) / len(kept), WORDS, 220 / seconds))
        d.model.close()


if __name__ == "__main__":
    main()
