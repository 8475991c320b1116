"""An attention layer as a generating transformer runs it: low-bit residual-expanded projections, keys and values in a 4-bit paged
cache, a packed batch of prompts first and then single tokens.

    python examples/attention_layer.py

prints, for the prompts and for every generated token, how far the layer's output is from the same layer with fp64 attention over
the full-precision keys and values (the error of 4 bits) and over the values that the cache holds (the error of the kernels).
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2311_15806_amd.binding as pipe  # noqa: E402


class AttentionLayer:
    """Projections of `width` features into heads query and kv_heads key/value heads and back, all expanded to K orders of 8-bit codes;
    the cache and the tables of up to `requests` requests."""

    def __init__(self, width, heads, kv_heads, head_dim, requests, pages, page_size, table_width, seed=0, K=2):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        W = torch.randn((heads + 2 * kv_heads) * head_dim, width, generator=g, device="cuda") * width ** -0.5
        self.qkv = pipe.pipe_expand(W, 8, K, 1.0, 16)
        self.out = pipe.pipe_expand(torch.randn(width, heads * head_dim, generator=g, device="cuda") * (heads * head_dim) ** -0.5, 8, K, 1.0, 16)
        self.heads, self.kv_heads, self.head_dim, self.page_size = heads, kv_heads, head_dim, page_size
        self.cache = torch.empty((pages, pipe.pipe_cache_page_bytes(kv_heads, head_dim, page_size)), dtype=torch.uint8, device="cuda")
        self.table = torch.full((requests, table_width), -1, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(pages, generator=g, device="cuda").int()
        self.used = torch.zeros(3, dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros(requests, dtype=torch.int32, device="cuda")

    def _step(self, x, fresh):
        """Tables, projection and cache of the fresh tokens x [tokens, width], fresh [requests] of each request."""
        self.lengths, starts, slots, _, self.used = pipe.pipe_cache_plan(self.lengths, fresh, self.page_size, self.free, self.used,
                                                                         self.table, x.shape[0])
        h = pipe.pipe_forward(self.qkv, x).view(x.shape[0], -1, self.head_dim)
        q, k, v = h.split([self.heads, self.kv_heads, self.kv_heads], dim=1)       # slices: no copies
        pipe.pipe_cache_write(k, v, slots, self.cache, self.page_size)
        return q, k, v, starts, slots

    def prompts(self, x, fresh):
        """The layer over packed prompts, which attend to themselves in full precision."""
        q, k, v, starts, slots = self._step(x, fresh)
        y = pipe.pipe_prompt_attention(q, k, v, starts)
        return pipe.pipe_forward(self.out, y.view(x.shape[0], -1)), (q, k, v, slots)

    def tokens(self, x, fresh, longest=0):
        """The layer over the next tokens of every request, which attend to the cache."""
        q, k, v, starts, slots = self._step(x, fresh)
        y = pipe.pipe_cache_attention(q, starts, self.lengths, self.cache, self.table, self.page_size, self.kv_heads, max_length=longest)
        return pipe.pipe_forward(self.out, y.view(x.shape[0], -1)), (q, k, v, slots)

    def held(self, slots):
        return pipe.pipe_cache_read(slots, self.cache, self.page_size, self.kv_heads, self.head_dim)


def reference(layer, q, keys, values):
    """One request's queries q [n, heads, head_dim], the last tokens of its keys and values, in fp64."""
    n, m, G = q.shape[0], keys.shape[0], layer.heads // layer.kv_heads
    k, v = (t.double().repeat_interleave(G, dim=1) for t in (keys, values))
    S = (q.double().transpose(0, 1) @ k.permute(1, 2, 0).contiguous()) * layer.head_dim ** -0.5
    late = torch.arange(m, device=q.device)[None] > m - n + torch.arange(n, device=q.device)[:, None]
    o = torch.softmax(S.masked_fill(late, float("-inf")), dim=-1) @ v.transpose(0, 1).contiguous()
    return o.transpose(0, 1).reshape(n, -1).float()


def main(steps=8, lens=(37, 1, 200, 96), width=1024, heads=16, kv_heads=4, head_dim=64, page_size=16, say=print):
    """Returns (error of the prompts, errors of the steps against full precision, errors of the steps against the cache's values)."""
    B = len(lens)
    layer = AttentionLayer(width, heads, kv_heads, head_dim, B, 64, page_size, 32)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")     # noqa: E731
    far = lambda a, b: float((a - b).norm() / b.norm())                    # noqa: E731

    x = torch.randn(sum(lens), width, generator=g, device="cuda")
    y, (q, k, v, slots) = layer.prompts(x, ints(lens))
    parts = [t.split(list(lens)) for t in (q, k, v, slots)]
    want = torch.cat([reference(layer, *(p[b] for p in parts[:3])) for b in range(B)])
    prompt_error = far(y, pipe.pipe_forward(layer.out, want))
    say("prompts of %s tokens: %.1e" % (list(lens), prompt_error))

    keys, values, places = ([p[b] for b in range(B)] for p in parts[1:])
    full, held = [], []
    for step in range(steps):
        x = torch.randn(B, width, generator=g, device="cuda")
        y, (q, k, v, slots) = layer.tokens(x, ints([1] * B), longest=max(lens) + step + 1)
        for b in range(B):
            keys[b], values[b] = torch.cat([keys[b], k[b:b + 1]]), torch.cat([values[b], v[b:b + 1]])
            places[b] = torch.cat([places[b], slots[b:b + 1]])
        want = torch.cat([reference(layer, q[b:b + 1], keys[b], values[b]) for b in range(B)])
        want4 = torch.cat([reference(layer, q[b:b + 1], *layer.held(places[b])) for b in range(B)])
        full.append(far(y, pipe.pipe_forward(layer.out, want)))
        held.append(far(y, pipe.pipe_forward(layer.out, want4)))
        say("token %d: %.1e of the full-precision layer, %.1e of the layer on the cache's values" % (step, full[-1], held[-1]))
    missing = int(layer.used[1])
    assert missing == 0, "the pool of pages is too small"
    return prompt_error, full, held


if __name__ == "__main__":
    main()
