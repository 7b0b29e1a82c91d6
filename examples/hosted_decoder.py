"""Coded serving of a hosted decoder: encode -> W workers' decoder over a paged cache -> decode, prompts and then token by token.

    python examples/hosted_decoder.py

A query is a sequence of embeddings (the encoder mixes real vectors, so a coded query is a mixture of K sequences, position
by position).  Every worker hosts the same decoder; here one GPU plays all of them, W * G coded sequences in one batch.  The
decoder's layers run on the three operators of hosted models:

    approxifer_linear         the projections with their bias, activation and residual, and the head, whose fp32 predictions
                              approxifer_decode takes as they are
    approxifer_qk_norm_rope   per-head norm and rotation of queries and keys, keys and values into the cache's pages
    approxifer_attention      a sliding window and a few first tokens that stay visible; pages that have left the window are
                              freed and given to the tokens that come
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2109_09868_b200 as ap  # noqa: E402


class HostedDecoder:
    """A decoder of `layers` layers (seeded random weights) with a paged cache for `sequences` sequences."""

    def __init__(self, sequences, longest, layers=2, width=256, heads=8, kv_heads=2, head=32, classes=10, window=0, sinks=0, page=16, seed=0, device="cuda"):
        self.heads, self.kv_heads, self.head, self.window, self.sinks, self.page = heads, kv_heads, head, window, sinks, page
        g = torch.Generator().manual_seed(seed)

        def weight(n, k):
            return (torch.randn((n, k), generator=g) / math.sqrt(k)).to(device, torch.bfloat16)

        def vector(n, mean):
            return (mean + 0.1 * torch.randn(n, generator=g)).to(device, torch.bfloat16)

        q, kv = heads * head, kv_heads * head
        self.layers = [dict(qkv=weight(q + 2 * kv, width), qkv_bias=vector(q + 2 * kv, 0.0), q_norm=vector(head, 1.0), k_norm=vector(head, 1.0),
                            out=weight(width, q), up=weight(4 * width, width), up_bias=vector(4 * width, 0.0), down=weight(width, 4 * width))
                       for _ in range(layers)]
        self.classes = weight(classes, width)
        angle = torch.arange(longest, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, head, 2, dtype=torch.float64) / head)
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], dim=1).float().to(device)
        # the cache of all layers, and whose pages are whose (kept on the host, sent with every step)
        per = (longest + page - 1) // page
        pages = sequences * per
        self.cache = [[torch.empty((pages, kv_heads, page, head), dtype=torch.bfloat16, device=device) for _ in range(2)] for _ in range(layers)]
        self.free = list(range(pages))
        self.table = torch.full((sequences, per), -1, dtype=torch.int32)
        self.length = torch.zeros(sequences, dtype=torch.int32)

    def _place(self, tokens):
        """Gives pages to the next `tokens` tokens of every sequence, after freeing those that no token to come will see."""
        if self.window:
            for b, n in enumerate(self.length.tolist()):
                gone = max(0, n + 1 - self.window) // self.page  # pages wholly before the window of the next token
                for p in range((self.sinks + self.page - 1) // self.page, gone):
                    if self.table[b, p] >= 0:
                        self.free.append(int(self.table[b, p]))
                        self.table[b, p] = -1
        at = self.length[:, None] + torch.arange(tokens, dtype=torch.int32)
        for b in range(len(self.length)):
            for p in range(int(at[b, 0]) // self.page, int(at[b, -1]) // self.page + 1):
                if self.table[b, p] < 0:
                    self.table[b, p] = self.free.pop()
        slots = self.table.gather(1, (at // self.page).long()).long() * self.page + at % self.page
        self.length += tokens
        return at.reshape(-1), slots.reshape(-1)

    def __call__(self, x):
        """bfloat16 embeddings [sequences][tokens][width], the tokens after those seen so far -> fp32 predictions
        [sequences][classes] of the last token."""
        sequences, tokens, width = x.shape
        positions, slots = (t.to(x.device) for t in self._place(tokens))
        table, length = self.table.to(x.device), self.length.to(x.device)
        start = torch.arange(0, (sequences + 1) * tokens, tokens, dtype=torch.int32, device=x.device)
        q, kv = self.heads * self.head, self.kv_heads * self.head
        h = x.reshape(-1, width)
        for w, (k_cache, v_cache) in zip(self.layers, self.cache):
            parts = ap.approxifer_linear(h, w["qkv"], bias=w["qkv_bias"]).split([q, kv, kv], dim=1)
            queries, keys, values = (p.unflatten(1, (-1, self.head)) for p in parts)
            queries = ap.approxifer_qk_norm_rope(queries, keys, values, w["q_norm"], w["k_norm"], self.cos_sin, positions, k_cache, v_cache, slots)
            seen = ap.approxifer_attention(queries, k_cache, v_cache, table, start, length, tokens, window=self.window, sinks=self.sinks)
            h = ap.approxifer_linear(seen.flatten(1), w["out"], residual=h)
            h = ap.approxifer_linear(ap.approxifer_linear(h, w["up"], bias=w["up_bias"], activation="gelu"), w["down"], residual=h)
        last = h.view(sequences, tokens, width)[:, -1]
        return ap.approxifer_linear(last, self.classes, out_dtype=torch.float32)


def main():
    K, W, G, tokens, steps, width, classes = 4, 6, 2, 50, 40, 256, 10
    params = ap.make_params(K, W)
    g = torch.Generator(device="cuda").manual_seed(1)
    decoder = HostedDecoder(G * W, tokens + steps, width=width, classes=classes, window=32, sinks=4)
    for step in range(steps + 1):
        n = tokens if step == 0 else 1
        queries = torch.randn((G, K, n * width), device="cuda", generator=g).bfloat16()
        coded = ap.approxifer_encode_bf16(params, queries)                   # [G][W][n * width]
        answers = decoder(coded.view(G * W, n, width)).view(G, W, classes)   # every worker's prediction
        mask = torch.full((G,), (1 << W) - 1 - (1 << (step % W)), dtype=torch.int32, device="cuda")  # one straggler, another each step
        predictions = ap.approxifer_decode(params, answers, mask)            # [G][K][classes]
        if step in (0, 1, steps):
            print("step %2d: %2d token(s) a sequence, %d free pages, predictions %s, first: %s"
                  % (step, n, len(decoder.free), tuple(predictions.shape), [round(v, 3) for v in predictions[0, 0, :4].tolist()]))


if __name__ == "__main__":
    main()
