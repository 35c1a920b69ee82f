"""A layout served with keys and queries rotated to their positions, from a cache
of 16 bits and of 4: rotated appends of every trie level, prefills over them, the
cached prompts read back, and a decode step that reads shared chunks once."""
import numpy as np
import pytest
import torch

from kv_reference import UNIT, attention, attention_bounds, close
from mx4_reference import partners, rotated
from paper_2609_13692_amd import mpt, serve
from paper_2609_13692_amd import workloads as wl

pytestmark = pytest.mark.gpu

HEADS, KV_HEADS, DIM = 6, 2, 64


def f64(x):
    return x.double().cpu().numpy()


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def at_positions(server, q, positions):
    """Queries rotated and rounded, checked against the definition."""
    freq = server.freq.cpu().numpy()
    got = server.cache.append_rotated(0, None, None, None, None, server.freq, q=q, interleaved=server.interleaved,
                                      positions=ints(positions))
    want = rotated(f64(q), positions, freq, server.interleaved)
    limit = UNIT[torch.bfloat16] * np.abs(want) + 2.0 ** -21 * partners(f64(q), freq, server.interleaved) + 1e-40
    close(f64(got), want, limit, "queries")
    return f64(got)


def check_cached(got, want, spread, bits):
    """Keys or values that the cache holds: rounded to bfloat16, or to codes of
    blocks of 32, whose steps are at most 2 * 2^e (and what passes the largest
    code is cut by at most 2^e), the largest element above 3.5 * 2^e. spread: 32-bit
    errors before that."""
    if bits == 16:
        limit = UNIT[torch.bfloat16] * np.abs(want) + spread
    else:
        top = (np.abs(want) + spread).reshape(*want.shape[:-1], -1, 32).max(-1)
        limit = np.repeat(top, 32, -1) / 3.5 + spread
    close(got, want, limit + 1e-38, "cached rows")


@pytest.mark.parametrize("page_size,interleaved,bits", [(1, False, 16), (16, True, 16), (16, False, 4), (1, True, 4), (128, False, 4)])
def test_served_layout(page_size, interleaved, bits):
    inst = wl.from_sets([[0, 1], [0, 1, 2], [0], [2, 1], [], [0, 1], [3, 0, 2]], [17, 33, 5, 130], name="prefixes of each other")
    project = serve.random_projection(inst, HEADS, KV_HEADS, DIM, torch.bfloat16, 1)
    freq = 100.0 ** (torch.arange(24, device="cuda") / -24)            # 48 of the 64 elements
    for seqs in (mpt.solve(inst)["orders"], inst.req_chunks):
        trie = serve.trie_of(inst.req_off, seqs, inst.weights)
        server = serve.LayoutServer(trie, project, HEADS, KV_HEADS, DIM, page_size=page_size, freq=freq,
                                    interleaved=interleaved, bits=bits)
        untouched = {c: tuple(x.clone() for x in project(c)) for c in range(len(inst.weights))}
        assert server.prefill(keep_depth=1) == int(server.new_tokens.sum())
        g = torch.Generator(device="cuda").manual_seed(3)
        q = torch.randn((inst.m, HEADS, DIM), device="cuda", generator=g).to(torch.bfloat16)
        out, lse = server.decode(q)
        assert server.cache.take_status() == []
        for c, parts in untouched.items():
            assert all(torch.equal(a, b) for a, b in zip(parts, project(c)))
        for i, (a, b) in enumerate(zip(inst.req_off[:-1], inst.req_off[1:])):
            chunks = [project(int(c)) for c in seqs[a:b]]
            if not chunks:
                assert not out[i].any() and torch.isinf(lse[i]).all()
                continue
            qs, ks, vs = (torch.cat(x) for x in zip(*chunks))
            length, leaf = len(ks), int(trie.leaf[i])
            k, v = (f64(x) for x in server.cache.read(0, ints([0, length]), ints([leaf]), length))
            want = rotated(f64(ks), range(length), freq.cpu().numpy(), interleaved)
            check_cached(k, want, 2.0 ** -21 * partners(f64(ks), freq.cpu().numpy(), interleaved), bits)
            check_cached(v, f64(vs), 0.0, bits)
            ref = attention(at_positions(server, q[i:i + 1], [length]), k, v, length - 1, causal=False)
            bo, bl = attention_bounds(*ref, length, DIM, torch.bfloat16, torch.bfloat16)
            close(f64(out[i:i + 1]), ref[0], bo, f"decode of request {i}")
            close(f64(lse[i:i + 1]), ref[1], bl, f"lse of request {i}")
            n = len(chunks[-1][0])
            ref = attention(at_positions(server, qs[-n:].contiguous(), range(length - n, length)), k, v, length - n)
            bo, _ = attention_bounds(*ref, length, DIM, torch.bfloat16, torch.bfloat16)
            close(f64(server.outputs[leaf]), ref[0], bo, f"prefill of request {i}")


@pytest.mark.parametrize("argv", [[], ["--rotate", "--bits", "4"]], ids=["plain", "rotated4"])
def test_the_command(argv, capsys):
    serve.main(argv)
    assert "decode step of 12 requests" in capsys.readouterr().out
