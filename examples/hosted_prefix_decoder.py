"""Coded serving of a hosted decoder whose queries begin alike, with weights held in 4 bits.

    python examples/hosted_prefix_decoder.py

The K queries of a group begin with the same prompt.  The encoder's weights of a coded query sum to one, so the W coded queries
begin with that prompt too: its keys and values are computed once, lie in the workers' cache once, and are read once for all the
sequences of a step.  Only what follows the prompt is encoded.  One GPU plays all workers, G * W sequences in one batch.  Beside
the operators of hosted_decoder.py a layer runs on

    approxifer_block_norm        between two blocks: the norm of a block's output, its gate, the residual (held in fp32), the norm
                                 before the next block
    approxifer_mx_linear         the projections, weights and activations in the 4-bit microscaled form (approxifer_mx_quantize
                                 makes that of the weights once)
    approxifer_prefix_attention  the common prompt and each sequence's own tokens
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2109_09868_b200 as ap  # noqa: E402


class PrefixDecoder:
    """A decoder of `layers` layers (seeded random weights) with a paged cache for a prompt of `prefix` tokens and `sequences`
    sequences of up to `longest` tokens behind it.  `ops`: whose operators it calls."""

    def __init__(self, sequences, prefix, longest, layers=2, width=256, heads=8, kv_heads=2, head=32, classes=10, page=16, seed=0, device="cuda", ops=ap):
        self.ops, self.heads, self.kv_heads, self.head, self.page, self.prefix = ops, heads, kv_heads, head, page, prefix
        g = torch.Generator().manual_seed(seed)

        def weight(n, k):
            return (torch.randn((n, k), generator=g) / math.sqrt(k)).to(device, torch.bfloat16)

        def vector(n, mean):
            return (mean + 0.1 * torch.randn(n, generator=g)).to(device, torch.bfloat16)

        q, kv = heads * head, kv_heads * head
        self.layers = [dict(qkv=ops.approxifer_mx_quantize(weight(q + 2 * kv, width)), q_norm=vector(head, 1.0), k_norm=vector(head, 1.0),
                            out=ops.approxifer_mx_quantize(weight(width, q)), up=ops.approxifer_mx_quantize(weight(4 * width, width)), up_bias=vector(4 * width, 0.0),
                            down=ops.approxifer_mx_quantize(weight(width, 4 * width)), before=[vector(width, 1.0) for _ in range(2)],
                            after=[vector(width, 1.0) for _ in range(2)], gate=[vector(width, 1.0) for _ in range(2)]) for _ in range(layers)]
        self.last_norm, self.classes = vector(width, 1.0), weight(classes, width)
        angle = torch.arange(prefix + longest, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, head, 2, dtype=torch.float64) / head)
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], dim=1).float().to(device)
        # pages: first the prompt's, then each sequence's
        first, per = (prefix + page - 1) // page, (longest + page - 1) // page
        self.cache = [[torch.empty((first + sequences * per, kv_heads, page, head), dtype=torch.bfloat16, device=device) for _ in range(2)] for _ in range(layers)]
        self.prefix_table = torch.arange(first, dtype=torch.int32, device=device)
        self.table = first + torch.arange(sequences * per, dtype=torch.int32, device=device).view(sequences, per)
        self.length = 0  # tokens of every sequence so far

    def _run(self, x, table, seen, before):
        """Embeddings [sequences][tokens][width] at the positions from `before` + `seen` on, their pages given by `table`, behind a
        prefix of `before` tokens -> the normed stream [sequences * tokens][width]."""
        ops, (sequences, tokens, width) = self.ops, x.shape
        dev, n = x.device, sequences * tokens
        at = seen + torch.arange(tokens, dtype=torch.int32, device=dev).expand(sequences, tokens)
        slots = (table.gather(1, (at // self.page).long()).long() * self.page + at % self.page).reshape(-1)
        positions = (before + at).reshape(-1).contiguous()
        start = torch.arange(0, n + 1, tokens, dtype=torch.int32, device=dev)
        length = torch.full((sequences,), seen + tokens, dtype=torch.int32, device=dev)
        q, kv = self.heads * self.head, self.kv_heads * self.head
        stream = x.reshape(n, width).float()
        stream, h = ops.approxifer_block_norm(stream, next_weight=self.layers[0]["before"][0])
        for i, (w, (k_cache, v_cache)) in enumerate(zip(self.layers, self.cache)):
            parts = ops.approxifer_mx_linear(h, *w["qkv"]).split([q, kv, kv], dim=1)
            queries, keys, values = (p.unflatten(1, (-1, self.head)) for p in parts)
            queries = ops.approxifer_qk_norm_rope(queries, keys, values, w["q_norm"], w["k_norm"], self.cos_sin, positions, k_cache, v_cache, slots)
            seen_by = ops.approxifer_prefix_attention(queries, k_cache, v_cache, self.prefix_table, before, table, start, length, tokens)
            out = ops.approxifer_mx_linear(seen_by.flatten(1), *w["out"])
            stream, h = ops.approxifer_block_norm(stream, out, gate=w["gate"][0], block_weight=w["after"][0], after="rms", gate_activation="sigmoid",
                                                  next_weight=w["before"][1], residual_out=stream)
            out = ops.approxifer_mx_linear(ops.approxifer_mx_linear(h, *w["up"], bias=w["up_bias"], activation="gelu_tanh"), *w["down"])
            following = self.layers[i + 1]["before"][0] if i + 1 < len(self.layers) else self.last_norm
            stream, h = ops.approxifer_block_norm(stream, out, gate=w["gate"][1], block_weight=w["after"][1], after="rms", gate_activation="sigmoid",
                                                  next_weight=following, residual_out=stream)
        return h

    def prompt(self, x):
        """The common prompt's embeddings [prefix][width], before the sequences' own."""
        self._run(x[None], self.prefix_table[None], 0, 0)

    def __call__(self, x):
        """bfloat16 embeddings [sequences][tokens][width], the tokens after those seen so far -> fp32 predictions
        [sequences][classes] of the last token."""
        sequences, tokens, width = x.shape
        h = self._run(x, self.table, self.length, self.prefix)
        self.length += tokens
        return self.ops.approxifer_linear(h.view(sequences, tokens, width)[:, -1], self.classes, out_dtype=torch.float32)


def main():
    K, W, G, prefix, tokens, steps, width, classes = 4, 6, 2, 200, 20, 30, 256, 10
    params = ap.make_params(K, W)
    g = torch.Generator(device="cuda").manual_seed(1)
    decoder = PrefixDecoder(G * W, prefix, tokens + steps, width=width, classes=classes)
    decoder.prompt(torch.randn((prefix, width), device="cuda", generator=g).bfloat16())
    for step in range(steps + 1):
        n = tokens if step == 0 else 1
        queries = torch.randn((G, K, n * width), device="cuda", generator=g).bfloat16()
        coded = ap.approxifer_encode_bf16(params, queries)                   # [G][W][n * width]
        answers = decoder(coded.view(G * W, n, width)).view(G, W, classes)   # every worker's prediction
        mask = torch.full((G,), (1 << W) - 1 - (1 << (step % W)), dtype=torch.int32, device="cuda")  # one straggler, another each step
        predictions = ap.approxifer_decode(params, answers, mask)            # [G][K][classes]
        if step in (0, 1, steps):
            print("step %2d: %2d token(s) a sequence behind %d, predictions %s, first: %s"
                  % (step, n, prefix, tuple(predictions.shape), [round(v, 3) for v in predictions[0, 0, :4].tolist()]))


if __name__ == "__main__":
    main()
