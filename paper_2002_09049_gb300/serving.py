"""An attention block served in few bits: the projections as microscaled 4-bit layers, keys and values in a
quantized paged cache, and the attention of new tokens over it.

``FewBitAttention`` owns the packed weights, the cache and the buffers of a decode step (kept for every batch
size and stream that it has met), so that a step allocates nothing: quantise the inputs, project (queries, keys and values in one product), write the
new tokens' keys and values, attend, quantise, project back -- six calls on one stream, or one graph
replay (``capture``).  ``prompt`` enters whole prompts into the cache, ``tokens`` reads slots back.

    python -m paper_2002_09049_gb300.serving      # one decode step's time, some batch sizes
"""
from __future__ import annotations

import contextlib

import torch

from . import binding


def _on(stream, device):
    """Makes `stream` the current one (None: it stays): what is allocated meanwhile belongs to it."""
    if stream is None:
        return contextlib.nullcontext()
    if not hasattr(stream, "wait_stream"):           # a handle that is not torch's
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device)
    return torch.cuda.stream(stream)


class FewBitAttention:
    def __init__(self, w_qkv, w_out, q_heads: int, heads: int, dim: int, pages: int, page: int = 64,
                 bits: int = 8, dtype=torch.bfloat16):
        """w_qkv [(q_heads + 2 heads) dim][d], w_out [d][q_heads dim]: the projections' weights on the
        device, quantised here.  The cache holds pages * page tokens in `bits` bits; dtype (fp16 or
        bf16) is that of inputs and outputs."""
        rows = (q_heads + 2 * heads) * dim
        if w_qkv.shape[0] != rows or w_out.shape[1] != q_heads * dim:
            raise ValueError(f"w_qkv must have {rows} rows and w_out {q_heads * dim} columns")
        self.q_heads, self.heads, self.dim, self.dtype = q_heads, heads, dim, dtype
        self.d, self.device = w_qkv.shape[1], w_qkv.device
        self.qkv_layout = binding.mpq_mx_layout(rows, self.d)
        self.out_layout = binding.mpq_mx_layout(w_out.shape[0], q_heads * dim)
        self.w_qkv = binding.mpq_mx_quantize(w_qkv, self.qkv_layout)
        self.w_out = binding.mpq_mx_quantize(w_out, self.out_layout)
        self.cache = binding.mpq_cache_layout(pages, page, heads, dim, bits)
        self.codes, self.scales = binding.mpq_cache_empty(self.cache, self.device)
        self._buffers, self._workspaces = {}, {}

    def _make_buffers(self, B):
        """What a step of B tokens writes on its way."""
        mk = lambda *shape: torch.empty(shape, dtype=self.dtype, device=self.device)
        x, o = binding.mpq_mx_layout(B, self.d), binding.mpq_mx_layout(B, self.q_heads * self.dim)
        packed = [torch.empty(lay.bytes, dtype=torch.uint8, device=self.device) for lay in (x, o)]
        return dict(x=x, o=o, x_packed=packed[0], o_packed=packed[1], qkv=mk(B, self.qkv_layout.rows),
                    attended=mk(B, self.q_heads, self.dim), y=mk(B, self.out_layout.rows))

    def _make_workspace(self):
        return torch.zeros(binding.MPQ_CACHE_WORKSPACE, dtype=torch.uint8, device=self.device)

    def _step_buffers(self, B):
        """The buffers of steps of B tokens on the current stream and its workspace, kept by stream (steps of
        one stream follow one another; those of two may overlap).  A graph being captured gets its own."""
        if torch.cuda.is_current_stream_capturing():
            return self._make_buffers(B), self._make_workspace()
        stream = torch._C._cuda_getCurrentRawStream(self.device.index)
        if stream not in self._workspaces:
            self._workspaces[stream] = self._make_workspace()
        if (B, stream) not in self._buffers:
            self._buffers[B, stream] = self._make_buffers(B)
        return self._buffers[B, stream], self._workspaces[stream]

    def _project(self, x, b):
        """Queries, keys and values [B][heads of each][dim] of inputs x [B][d] (views of one buffer)."""
        binding.mpq_mx_quantize(x, b["x"], b["x_packed"])
        binding.mpq_mx_linear(b["x_packed"], b["x"], self.w_qkv, self.qkv_layout, Y=b["qkv"])
        rows = b["qkv"].view(x.shape[0], self.q_heads + 2 * self.heads, self.dim)
        return rows.split((self.q_heads, self.heads, self.heads), 1)

    def prompt(self, x, slots, stream=None):
        """Enters tokens x [T][d] into the cache at slots [T] (int64).  Its buffers are allocated for the
        call, on the stream that it runs on."""
        with _on(stream, self.device):
            _, k, v = self._project(x, self._make_buffers(x.shape[0]))
            binding.mpq_cache_write(k, v, slots, self.cache, self.codes, self.scales)

    def step(self, x, slots, table, lens, window: int = 0, stream=None):
        """One new token of every sequence: x [B][d], its slot in the cache (int64 [B]), the
        sequences' pages (int32 [B][columns]) and lengths with the new token (int32 [B]).  Returns the
        block's outputs [B][d] (a buffer that the next step of B tokens on the same stream overwrites)."""
        with _on(stream, self.device):
            return self._step(x, slots, table, lens, window, *self._step_buffers(x.shape[0]))

    def _step(self, x, slots, table, lens, window, b, workspace):
        q, k, v = self._project(x, b)
        binding.mpq_cache_write(k, v, slots, self.cache, self.codes, self.scales)
        binding.mpq_cache_attention(q, table, lens, self.cache, self.codes, self.scales,
                                    window=window, O=b["attended"], workspace=workspace)
        binding.mpq_mx_quantize(b["attended"].view(x.shape[0], -1), b["o"], b["o_packed"])
        return binding.mpq_mx_linear(b["o_packed"], b["o"], self.w_out, self.out_layout, Y=b["y"])

    def tokens(self, slots, stream=None):
        """The keys and values [T][heads][dim] that the cache holds at slots [T]."""
        return binding.mpq_cache_read(slots, self.cache, self.codes, self.scales, dtype=self.dtype,
                                      stream=stream)

    def capture(self, B: int, columns: int, window: int = 0):
        """A CUDA graph of one step for B sequences of up to `columns` pages: its inputs are the
        returned object's x, slots, table and lens, filled before replay().  It has buffers and a workspace
        of its own and keeps the block; one graph's replays follow one another."""
        return CapturedStep(self, B, columns, window)


class CapturedStep:
    def __init__(self, block: FewBitAttention, B: int, columns: int, window: int = 0):
        mk = lambda shape, dtype: torch.zeros(shape, dtype=dtype, device=block.device)
        self.x = mk((B, block.d), block.dtype)
        self.slots = mk((B,), torch.int64).fill_(-1)      # no slot, no tokens: the warm-up writes nothing
        self.table = mk((B, columns), torch.int32)
        self.lens = mk((B,), torch.int32)
        self.block = block                # the graph reads its weights and its cache
        self._buffers, self._workspace = block._make_buffers(B), block._make_workspace()
        args = (self.x, self.slots, self.table, self.lens, window, self._buffers, self._workspace)
        side = torch.cuda.Stream(block.device)
        side.wait_stream(torch.cuda.current_stream(block.device))
        with torch.cuda.stream(side):
            block._step(*args)
        torch.cuda.current_stream(block.device).wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.y = block._step(*args)

    def replay(self):
        """Enqueues the step on the current stream; returns its outputs' buffer."""
        self.graph.replay()
        return self.y


def main():
    dev = torch.device("cuda:0")
    d, q_heads, heads, dim, page, length = 4096, 32, 8, 128, 64, 2048
    gen = torch.Generator(device=dev).manual_seed(1)
    w = lambda rows, cols: 0.02 * torch.randn(rows, cols, generator=gen, device=dev)
    for B in (1, 8, 64):
        per = length // page
        block = FewBitAttention(w((q_heads + 2 * heads) * dim, d), w(d, q_heads * dim), q_heads, heads,
                                dim, pages=B * per, page=page)
        for b in range(B):
            x = torch.randn(length, d, generator=gen, device=dev).to(torch.bfloat16)
            block.prompt(x, torch.arange(length, device=dev) + b * length)
        step = block.capture(B, per)
        step.x.copy_(torch.randn(B, d, generator=gen, device=dev))
        step.table.copy_(torch.arange(B * per, device=dev).view(B, per))
        step.lens.fill_(length)
        step.slots.copy_(torch.arange(1, B + 1, device=dev) * length - 1)
        for _ in range(5):
            step.replay()
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        for _ in range(50):
            step.replay()
        end.record()
        torch.cuda.synchronize()
        us = begin.elapsed_time(end) / 50 * 1e3
        print(f"{B:3d} sequences of {length} tokens: {us:.1f} us a step, "
              f"{B / us * 1e6:.0f} tokens/s through the block")


if __name__ == "__main__":
    main()
