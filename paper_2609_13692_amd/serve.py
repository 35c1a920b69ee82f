"""A layout served from a paged key/value cache.

The solver's layouts say in which order each request's chunks go, so that the
trie of all prompts is light; :class:`LayoutServer` holds that trie in a
:class:`.kv.KvCache`. Level by level every trie node becomes a sequence forked
off its parent: the parent's pages are shared, only the node's own chunk is
computed (its keys and values appended, its queries attended over the whole
prefix), so the tokens computed are the layout's trie cost (Eq. 1), which
``mpt_layout_cost`` bills. Nodes that no request ends at are freed once their
children exist, unless the prefill is told to keep their depth; their pages live
on in the children. Keys and queries can be rotated to their positions in the
request (a node's tokens have the same ones in all requests below it), and the
cache can be of 4 bits. It is a demonstration of the cache's calls: one layer, and a
decode step whose tokens are not appended.

``python -m paper_2609_13692_amd.serve`` runs a small retrieval-shaped instance
through the exact solver, the cache and a decode step in which each first
chunk's tokens are read once for all requests below it; ``--rotate`` rotates keys
and queries, ``--bits 4`` holds the cache in 4 bits.
"""
from __future__ import annotations

import argparse
import dataclasses

import numpy as np
import torch

from . import kv, mpt
from . import workloads as wl


@dataclasses.dataclass(frozen=True)
class Trie:
    """The nodes of a layout's trie, parents first; -1 is the root."""

    parent: np.ndarray       # int64 [nodes]
    chunk: np.ndarray        # int64 [nodes]
    depth: np.ndarray        # int64 [nodes], 1 for children of the root
    length: np.ndarray       # int64 [nodes]: tokens from the root to the node's end
    leaf: np.ndarray         # int64 [requests]: node that each request ends at


def trie_of(seq_off, seqs, weights) -> Trie:
    """The trie of the sequences seqs[seq_off[i] .. seq_off[i + 1])."""
    nodes, parent, chunk, depth, length, leaf = {}, [], [], [], [], []
    for a, b in zip(seq_off[:-1], seq_off[1:]):
        at = -1
        for c in seqs[a:b]:
            key = (at, int(c))
            if key not in nodes:
                nodes[key] = len(parent)
                parent.append(at)
                chunk.append(int(c))
                depth.append(1 if at < 0 else depth[at] + 1)
                length.append(int(weights[c]) + (0 if at < 0 else length[at]))
            at = nodes[key]
        leaf.append(at)
    order = np.argsort(np.asarray(depth, dtype=np.int64), kind="stable")
    new = np.empty(len(parent) + 1, dtype=np.int64)
    new[order], new[-1] = np.arange(len(parent)), -1
    pick = lambda x: np.asarray(x, dtype=np.int64)[order]  # noqa: E731
    return Trie(new[pick(parent)], pick(chunk), pick(depth), pick(length), new[np.asarray(leaf, dtype=np.int64)])


class LayoutServer:
    """A cache of one layer that holds the prompts of a layout.

    ``project(chunk)`` returns the queries [tokens, heads, dim], keys and
    values [tokens, kv_heads, dim] of a chunk's tokens on the device. With
    ``freq`` (float32 [pairs] on the device, see :meth:`.kv.KvCache.append_rotated`)
    queries and keys are rotated to their tokens' positions; ``bits`` are the
    cache's (16 or 4).
    """

    def __init__(self, trie: Trie, project, heads, kv_heads, dim, page_size=16, dtype=torch.bfloat16, device="cuda",
                 freq=None, interleaved=False, bits=16):
        self.freq, self.interleaved = freq, interleaved
        self.trie, self.project, self.heads, self.device = trie, project, heads, torch.device(device)
        tokens = trie.length - np.where(trie.parent < 0, 0, trie.length[trie.parent])
        self.new_tokens = tokens
        # a node's own pages: its tokens, and its parent's last page once more
        pages = int((-(-(tokens + page_size - 1) // page_size)).sum())
        self.cache = kv.KvCache.create(1, max(1, pages), page_size, kv_heads, dim, max(1, len(tokens)),
                                       int(trie.length.max(initial=1)) + page_size, dtype, device, bits=bits)
        self.outputs = {}                      # attention outputs of each node's tokens
        self.held = np.zeros(len(tokens), dtype=bool)   # nodes whose slots hold their prefix

    def _ints(self, x):
        return torch.as_tensor(np.asarray(x, dtype=np.int32), device=self.device)

    def prefill(self, keep_depth=0) -> int:
        """Computes every node, slot i for node i; returns the tokens
        computed. Nodes up to keep_depth keep their slots, so that decode can
        read them once for the requests below them."""
        t, computed = self.trie, 0
        ends = np.zeros(len(t.parent), dtype=bool)
        ends[t.leaf[t.leaf >= 0]] = True
        for d in range(1, int(t.depth.max(initial=0)) + 1):
            level = np.flatnonzero(t.depth == d)
            parent = t.parent[level]
            keep = np.where(parent < 0, 0, t.length[parent])
            self.cache.fork(self._ints(parent), self._ints(level), self._ints(keep), self._ints(t.length[level]), check=True)
            q, k, v = (torch.cat(x) for x in zip(*(self.project(int(t.chunk[i])) for i in level)))
            off = np.concatenate([[0], np.cumsum(self.new_tokens[level])])
            if self.freq is None:
                self.cache.append(0, k, v, self._ints(off), self._ints(level))
            else:
                self.cache.append_rotated(0, k, v, self._ints(off), self._ints(level), self.freq, q=q, q_out=q,
                                          interleaved=self.interleaved)
            out, _ = self.cache.attend(0, q, self._ints(off), self._ints(level))
            self.held[level] = True
            for i, a, b in zip(level, off, off[1:]):
                self.outputs[int(i)] = out[a:b]
            computed += int(off[-1])
            done = np.flatnonzero((t.depth == d - 1) & ~ends & (t.depth > keep_depth))
            if len(done):
                self.cache.free(self._ints(done))
                self.held[done] = False
        live = self.cache.compact(check=True)
        self.live_pages = live
        return computed

    def decode(self, q, shared_depth=1):
        """Attention of one query per request (q [requests, heads, dim], not
        appended, rotated to the position after the prompt) over its prompt. Nodes are read once for all requests below
        them: of each request the deepest up to shared_depth whose slot prefill
        kept (keep_depth); a request without one reads its whole prompt."""
        t, requests = self.trie, len(self.trie.leaf)
        if not self.held[t.leaf[t.leaf >= 0]].all():
            raise RuntimeError("prefill has not computed every prompt")
        first = t.leaf.copy()                  # the node whose tokens are read once, -1: none
        depth, held = np.append(t.depth, 0), np.append(self.held, True)     # the root's are the last
        while (up := (first >= 0) & ((depth[first] > shared_depth) | ~held[first])).any():
            first[up] = t.parent[first[up]]
        # requests by that node, those without one last; requests without chunks see nothing
        order = np.argsort(np.where(first < 0, len(t.parent), first), kind="stable")
        order = order[t.leaf[order] >= 0]
        shared = int((first[order] >= 0).sum())
        groups, counts = np.unique(first[order[:shared]], return_counts=True)
        pick = torch.as_tensor(order, device=self.device)
        sorted_q = q[pick].contiguous()
        if self.freq is not None:
            self.cache.append_rotated(0, None, None, None, None, self.freq, q=sorted_q, q_out=sorted_q,
                                      interleaved=self.interleaved, positions=self._ints(t.length[t.leaf[order]]))
        each = np.arange(len(order) + 1)
        begin = np.append(t.length, 0)[first[order]]
        out, lse = self.cache.attend(0, sorted_q, self._ints(each), self._ints(t.leaf[order]), causal=False,
                                     kv_begin=self._ints(begin), out_dtype=torch.float32)
        whole = torch.zeros((requests, self.heads, q.shape[2]), dtype=q.dtype, device=self.device)
        whole_lse = torch.full((requests, self.heads), -float("inf"), device=self.device)
        if shared:
            prefix, prefix_lse = self.cache.attend(0, sorted_q[:shared], self._ints(np.concatenate([[0], np.cumsum(counts)])),
                                                   self._ints(groups), causal=False, out_dtype=torch.float32)
            kv.merge([prefix, out[:shared]], [prefix_lse, lse[:shared]], out=out[:shared], lse=lse[:shared])
        whole[pick], whole_lse[pick] = out.to(q.dtype), lse
        return whole, whole_lse


def random_projection(inst, heads, kv_heads, dim, dtype, seed, device="cuda"):
    """Random queries, keys and values per chunk (the same wherever the chunk
    stands), in the place of a model's projections."""
    made = {}

    def project(chunk):
        if chunk not in made:
            g = torch.Generator(device=device).manual_seed(seed * 1000003 + chunk)
            n = int(inst.weights[chunk])
            made[chunk] = tuple(torch.empty((n, h, dim), device=device).normal_(generator=g).to(dtype)
                                for h in (heads, kv_heads, kv_heads))
        return made[chunk]

    return project


def main(argv=None) -> None:
    args = argparse.ArgumentParser(prog="python -m paper_2609_13692_amd.serve", description=__doc__.splitlines()[0])
    args.add_argument("--rotate", action="store_true", help="rotate keys and queries to their positions")
    args.add_argument("--bits", type=int, choices=(16, 4), default=16, help="of the cache's elements")
    args = args.parse_args(argv)
    freq = 10000.0 ** (torch.arange(64, device="cuda") / -64) if args.rotate else None
    inst = wl.gen_retrieval(m=12, u=200, topics=6, k=6, seed=1)
    orders = mpt.solve(inst)["orders"]
    trie = trie_of(inst.req_off, orders, inst.weights)
    server = LayoutServer(trie, random_projection(inst, 8, 2, 128, torch.bfloat16, 0), 8, 2, 128,
                          freq=freq, bits=args.bits)
    computed = server.prefill(keep_depth=1)
    total = int(sum(inst.weights[c] for c in orders))
    print(f"{inst.name}: {computed} of {total} prompt tokens computed, {len(trie.parent)} trie nodes, "
          f"{server.live_pages} pages of {server.cache.page_size} tokens in use")
    q = torch.randn((inst.m, 8, 128), device="cuda").to(torch.bfloat16)
    out, lse = server.decode(q)
    print(f"decode step of {inst.m} requests: outputs {tuple(out.shape)}, log sums {lse.min().item():.3f} .. {lse.max().item():.3f}")


if __name__ == "__main__":
    main()
