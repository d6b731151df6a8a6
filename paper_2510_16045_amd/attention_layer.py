"""The attention block of a decoder layer on packed weights and a 4-bit KV cache: how the library's calls go together.

    qkv = ams_linear(x);  ams_kv_write(k, v);  ams_kv_attention(q);  ams_linear(o)

q and k are used as the projection gives them: a model with rotary embeddings rotates them between the projection and ams_kv_write.
Projections of up to MAX_M rows run on the packed weights; those of prompts restore a matrix to fp16 once and multiply with the
library GEMM; captured ones of more rows run MAX_M rows at a time.  A decode step of fixed batch is captured as a HIP graph: the sequences' lengths lie on the GPU and grow from replay to
replay.  ``python -m paper_2510_16045_amd.attention_layer`` runs a prompt and decode steps of a Llama-3-8B-shaped block on
random weights and prints what a step takes.
"""

from __future__ import annotations

import numpy as np

from . import FP425, KV_WORKSPACE_BYTES, MAX_M, ams_dequant, ams_init, ams_kv_attention, ams_kv_cache, ams_kv_write, ams_linear, ams_pack, synth


class PackedLinear:
    """Y = X W^T on weights packed from host fp16 [N, K]."""

    def __init__(self, weights: np.ndarray, fmt: int = FP425):
        import torch

        packed, scales = ams_pack(fmt, weights)
        self.N, self.K, self.fmt = *weights.shape, fmt
        self.packed = torch.from_numpy(packed).cuda()
        self.scales = torch.from_numpy(scales.view(np.int16)).cuda().view(torch.float16)

    def __call__(self, x, out=None):
        import torch

        rows = x.shape[0]
        if rows <= MAX_M:
            return ams_linear(self.packed, self.scales, x, self.N, self.fmt, out=out)
        if torch.cuda.is_current_stream_capturing():
            # a graph holds kernels of this library alone: the library GEMM sets itself up at its first call, which ends the process where
            # that is captured
            y = torch.empty((rows, self.N), dtype=x.dtype, device=x.device) if out is None else out
            for i in range(0, rows, MAX_M):
                ams_linear(self.packed, self.scales, x[i : i + MAX_M], self.N, self.fmt, out=y[i : i + MAX_M])
            return y
        y = x @ ams_dequant(self.fmt, self.packed, self.scales, self.N, self.K).t()
        return y if out is None else out.copy_(y)


class AttentionLayer:
    """Projections, cache and attention of one layer; sequence b owns the pages block_table[b], int32 [batch, pages]."""

    def __init__(self, qkv: np.ndarray, o: np.ndarray, heads: int, kv_heads: int, n_pages: int, block_table, page_size: int = 64, scale_group: int = 32, fmt: int = FP425, workspace=None):
        import torch

        self.head_dim = qkv.shape[0] // (heads + 2 * kv_heads)
        self.heads, self.kv_heads, self.page_size, self.scale_group = heads, kv_heads, page_size, scale_group
        self.qkv, self.o = PackedLinear(qkv, fmt), PackedLinear(o, fmt)
        self.cache = ams_kv_cache(n_pages, kv_heads, self.head_dim, page_size, scale_group)
        self.block_table = block_table
        # one for all layers of a stream: their calls follow one another
        self.workspace = torch.zeros(KV_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda") if workspace is None else workspace

    def __call__(self, x, kv_lens, q_starts=None, max_q_len: int = None, out=None):
        """x fp16 [rows, hidden]: the last rows of sequences of kv_lens[b] tokens, these among them.

        max_q_len: the most rows of any of them, where the caller knows (drafts are faster with it)."""
        rows = self.qkv(x).view(-1, self.heads + 2 * self.kv_heads, self.head_dim)
        q, k, v = rows[:, : self.heads], rows[:, self.heads : self.heads + self.kv_heads], rows[:, self.heads + self.kv_heads :]
        ams_kv_write(self.cache, k, v, self.block_table, kv_lens, self.scale_group, q_starts=q_starts)
        y = ams_kv_attention(q, self.cache, self.block_table, kv_lens, self.scale_group, q_starts=q_starts, max_q_len=max_q_len, workspace=self.workspace)
        return self.o(y.view(-1, self.heads * self.head_dim), out=out)


class DecodeStep:
    """A decode step of a batch as a HIP graph: x in, y out; every replay adds a token to each sequence.

    A step for which a sequence has no place left in the block table is refused.  The host counts the steps from the lengths that it has
    seen, and looks at kv_lens again, which waits for the GPU, only where by that count there is no place; whoever makes a sequence
    longer by hand calls recount()."""

    def __init__(self, layer: AttentionLayer, kv_lens):
        import torch

        ams_init()
        batch, hidden = kv_lens.shape[0], layer.qkv.K
        self.layer, self.kv_lens = layer, kv_lens
        self.capacity = layer.block_table.shape[1] * layer.page_size
        self.recount()
        self.x = torch.zeros((batch, hidden), dtype=torch.float16, device="cuda")
        self.y = torch.zeros_like(self.x)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.kv_lens += 1
            layer(self.x, self.kv_lens, out=self.y)

    def recount(self):
        self.places = self.capacity - int(self.kv_lens.max())  # that the longest sequence has left

    def __call__(self, x):
        if self.places <= 0:
            self.recount()
        if self.places <= 0:
            raise ValueError(f"a sequence has no place for another token: the block table has room for {self.capacity}")
        self.places -= 1
        self.x.copy_(x)
        self.graph.replay()
        return self.y


def main(batch: int = 8, prompt: int = 2000, steps: int = 64, page_size: int = 64):
    import time

    import torch

    hidden, heads, kv_heads, dim = 4096, 32, 8, 128  # Llama-3-8B
    pages = -(-(prompt + steps + 1) // page_size)
    table = torch.arange(batch * pages, dtype=torch.int32, device="cuda").view(batch, pages)
    layer = AttentionLayer(synth.gaussian_weights((heads + 2 * kv_heads) * dim, hidden, 0), synth.gaussian_weights(hidden, heads * dim, 1), heads, kv_heads, batch * pages, table, page_size)
    lens = torch.full((batch,), prompt, dtype=torch.int32, device="cuda")
    starts = torch.arange(batch + 1, dtype=torch.int32, device="cuda") * prompt
    layer(torch.randn((batch * prompt, hidden), device="cuda").half(), lens, q_starts=starts, max_q_len=prompt)
    step = DecodeStep(layer, lens)
    x = torch.randn((batch, hidden), device="cuda").half()
    step(x)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(steps - 1):
        step(x)
    torch.cuda.synchronize()
    took = (time.perf_counter() - t) / (steps - 1)
    held = layer.cache.numel() / (batch * pages * page_size)
    print(f"batch {batch}, {prompt} tokens each and {steps} steps: {1e6 * took:.1f} us a step; the cache holds {held:.0f} bytes a token, fp16 would {4 * kv_heads * dim}")


if __name__ == "__main__":
    main()
