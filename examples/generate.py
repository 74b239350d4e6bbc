"""Attention of one layer with a 4-bit paged cache, as a serving program runs it.

    python examples/generate.py [--sequences 8] [--prompt 1000] [--tokens 64]

A `Layer` takes what the projection of a layer leaves, queries, keys and values side by side in one buffer, and returns what
attention makes of them: heads are normed and rotated by position (or rotated alone), keys and values go to pages of the cache in four bits,
and the queries attend to all that the cache holds of their sequence.  A prompt is one call; the tokens after it are a graph
that is captured once and replayed, since everything that changes from token to token lies in buffers on the GPU.
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1810_08723_amd as ocn  # noqa: E402

_NAMES = {torch.float16: "half", torch.bfloat16: "bfloat16", torch.float32: "float", torch.float64: "double", torch.int32: "int32",
          torch.uint8: "uint8"}


def view(t: torch.Tensor) -> ocn.Tensor:
    """The descriptor of a torch tensor: its address, type, sizes and byte strides"""
    e = t.element_size()
    return ocn.Tensor(t.data_ptr(), _NAMES[t.dtype], tuple(t.shape), tuple(n * e for n in t.stride()), 0, t.device.index or 0, t)


class Layer:
    def __init__(self, sequences, most_tokens, heads=32, kv_heads=8, channels=128, page=64, dtype=torch.bfloat16, norm=True, base=10000.0,
                 stretch="none", factor=1.0, original=0.0, device="cuda"):
        self.shape = sequences, heads, kv_heads, channels
        self.page, self.dtype, self.device = page, dtype, device
        columns = -(-most_tokens // page)
        # pages in no particular order, as an allocator that gives and takes them leaves them
        self.table = torch.randperm(sequences * columns, device=device).to(torch.int32).view(sequences, columns)
        self.cache = torch.zeros(sequences * columns, kv_heads, ocn.cache_block_bytes(page, channels), dtype=torch.uint8, device=device)
        self.length = torch.zeros(sequences, 1, dtype=torch.int32, device=device)
        frequencies, self.magnitude = ocn.rotary_frequencies(channels, base, stretch, factor, original)
        self.frequencies = torch.tensor(frequencies, dtype=torch.float64, device=device)
        self.weights = [torch.ones(channels, dtype=dtype, device=device) for _ in range(2)] if norm else None
        self.room = columns * page      # tokens that a sequence may still have
        self._graph = None

    def _take(self, tokens):
        if tokens > self.room:
            raise ValueError(f"{tokens} tokens, and pages for {self.room}")
        self.room -= tokens

    def _buffers(self, tokens):
        """What a call of so many tokens needs beside the cache, and its descriptors"""
        sequences, heads, kv, channels = self.shape
        b = {"qkv": torch.zeros(sequences, tokens, heads + 2 * kv, channels, dtype=self.dtype, device=self.device),
             "out": torch.zeros(sequences, tokens, heads, channels, dtype=self.dtype, device=self.device)}
        b["positions"], b["slots"], b["seen"] = (torch.zeros(sequences, tokens, dtype=torch.int32, device=self.device) for _ in range(3))
        v = {n: view(t) for n, t in b.items()}
        v["q"], v["k"], v["v"] = (view(t) for t in b["qkv"].split([heads, kv, kv], dim=2))
        v["table"], v["cache"] = view(self.table), view(self.cache)
        v["rotation"] = ocn.Rotation(v["positions"], view(self.frequencies), channels, "half", self.magnitude)
        b["steps"] = torch.arange(tokens, dtype=torch.int32, device=self.device)
        b["workspace"] = torch.empty(max(1, ocn.cache_attention_workspace_bytes(v["q"], v["cache"], v["table"])), dtype=torch.uint8, device=self.device)
        return b, v

    def _run(self, b, v):
        """The tokens in b["qkv"], after those that the cache holds"""
        torch.add(self.length, b["steps"], out=b["positions"])
        torch.add(b["positions"], 1, out=b["seen"])
        at = b["positions"].long()
        b["slots"].copy_(torch.gather(self.table, 1, at // self.page) * self.page + b["positions"] % self.page)
        if self.weights:
            q_weight, k_weight = (view(w) for w in self.weights)
            ocn.norm_rotary(v["q"], q_weight, v["q"], v["k"], k_weight, v["k"], rotation=v["rotation"])
            ocn.cache_append(v["k"], v["v"], v["slots"], v["cache"])
        else:
            ocn.rotary(v["q"], v["rotation"], v["q"])
            ocn.cache_append(v["k"], v["v"], v["slots"], v["cache"], rotation=v["rotation"])
        ocn.cache_attention(v["q"], v["cache"], v["table"], v["seen"], v["out"], 1 / math.sqrt(self.shape[3]), workspace=b["workspace"])
        self.length.add_(b["qkv"].shape[1])

    def prompt(self, qkv):
        """[sequences, tokens, heads + 2 kv_heads, channels] to [sequences, tokens, heads, channels]"""
        self._take(qkv.shape[1])
        b, v = self._buffers(qkv.shape[1])
        b["qkv"].copy_(qkv)
        self._run(b, v)
        return b["out"]

    def token(self, qkv):
        """The same for one token of each sequence; the result is overwritten by the next one"""
        self._take(1)
        if self._graph is None:
            self._one = self._buffers(1)
            length, table = self.length.clone(), self.table.clone()
            self.table.fill_(-1)        # one pass loads the kernels; its token goes nowhere
            self._run(*self._one)
            self.table.copy_(table)
            self.length.copy_(length)
            torch.cuda.synchronize()
            self._graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self._graph):
                self._run(*self._one)
        self._one[0]["qkv"].copy_(qkv)
        self._graph.replay()
        return self._one[0]["out"]


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--sequences", type=int, default=8)
    p.add_argument("--prompt", type=int, default=1000)
    p.add_argument("--tokens", type=int, default=64)
    a = p.parse_args()
    layer = Layer(a.sequences, a.prompt + a.tokens)
    make = lambda tokens: torch.randn(a.sequences, tokens, 48, 128, device="cuda").to(torch.bfloat16)  # noqa: E731
    layer.prompt(make(a.prompt))
    one = make(1)
    layer.token(one)
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(a.tokens - 1):
        layer.token(one)
    torch.cuda.synchronize()
    us = (time.perf_counter() - start) * 1e6 / max(1, a.tokens - 1)
    print(f"{a.sequences} sequences of {a.prompt} tokens in {layer.cache.numel() / 2**20:.1f} MiB of cache; a token of each: {us:.1f} us")


if __name__ == "__main__":
    main()
