"""A layout served from the paged cache: the tokens computed are the layout's
trie cost, and what comes out is attention over each request's whole prompt."""
import numpy as np
import pytest
import torch

from kv_reference import attention, attention_bounds, close
from paper_2609_13692_amd import mpt, serve
from paper_2609_13692_amd import workloads as wl

pytestmark = pytest.mark.gpu

HEADS, KV_HEADS, DIM = 6, 2, 64


def cost_of(inst, seqs):
    t = lambda x, dt: torch.as_tensor(np.asarray(x), dtype=dt, device="cuda")  # noqa: E731
    ws = mpt.alloc_layout_workspace(inst.m, inst.n_chunks, inst.nnz)
    return mpt.mpt_layout_cost(inst.m, inst.n_chunks, t(inst.weights, torch.int64), t(inst.req_off, torch.int64),
                               t(seqs, torch.int32), None, ws)


@pytest.mark.parametrize("page_size", [1, 16])
@pytest.mark.parametrize("inst", [
    wl.random_small(m=7, u=9, kmin=0, kmax=5, wmax=40, seed=3, allow_empty=True),
    wl.from_sets([[0, 1], [0, 1, 2], [0], [2, 1], [], [0, 1]], [17, 33, 5], name="prefixes of each other"),
], ids=["random", "prefixes"])
def test_served_layout(inst, page_size):
    """Requests of several lengths, empty ones and prefixes of others, laid
    out by the exact solver and as they come."""
    project = serve.random_projection(inst, HEADS, KV_HEADS, DIM, torch.bfloat16, 1)
    for seqs in (mpt.solve(inst)["orders"], inst.req_chunks):
        trie = serve.trie_of(inst.req_off, seqs, inst.weights)
        server = serve.LayoutServer(trie, project, HEADS, KV_HEADS, DIM, page_size=page_size)
        assert server.prefill(keep_depth=1) == cost_of(inst, seqs)
        assert server.live_pages == int((server.cache.ref > 0).sum())
        q = torch.randn((inst.m, HEADS, DIM), device="cuda").to(torch.bfloat16)
        out, lse = server.decode(q)
        assert server.cache.take_status() == []
        for i, (a, b) in enumerate(zip(inst.req_off[:-1], inst.req_off[1:])):
            chunks = [project(int(c)) for c in seqs[a:b]]
            if not chunks:
                assert not out[i].any() and torch.isinf(lse[i]).all()
                continue
            qs, k, v = (torch.cat(x).double().cpu().numpy() for x in zip(*chunks))
            ref = attention(q[i:i + 1].double().cpu().numpy(), k, v, len(k) - 1, causal=False)
            bo, bl = attention_bounds(*ref, len(k), DIM, torch.bfloat16, torch.bfloat16)
            close(out[i:i + 1].double().cpu().numpy(), ref[0], bo, f"decode of request {i}")
            close(lse[i:i + 1].double().cpu().numpy(), ref[1], bl, f"lse of request {i}")
            # the prefill of the request's last chunk, over its whole prefix
            n = len(chunks[-1][0])
            ref = attention(qs[-n:], k, v, len(k) - n)
            bo, _ = attention_bounds(*ref, len(k), DIM, torch.bfloat16, torch.bfloat16)
            close(server.outputs[int(trie.leaf[i])].double().cpu().numpy(), ref[0], bo, f"prefill of request {i}")
