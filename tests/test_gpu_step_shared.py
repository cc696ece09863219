"""Calls on one pool that share its workspace of cut contexts and its staging slots: different work on two streams and in two threads, none
of it waited for in between, each result the one of its own call alone."""
import threading

import numpy as np
import pytest
import torch

from oracle import step_oracle as so
from test_gpu_step import Setup, spread

pytestmark = pytest.mark.gpu

LONG = [(4000, 2), (3000, 3), (2500, 4), (3900, 1), (1200, 2), (3300, 2)]
SHORT = spread(470, 0, 40, [1], seed=3)


def batches(s, groups):
    """One call per group of the sequences: its arguments, and its result, checked against the oracle, with nothing else under way."""
    calls = []
    for group in groups:
        rows = np.concatenate([np.arange(s.cu[i], s.cu[i + 1]) for i in group])
        n = np.diff(s.cu)[group]
        where = (np.concatenate([[0], np.cumsum(n)]).astype(np.int32), s.P[group], s.t["tables"][torch.as_tensor(group).cuda()].contiguous())
        q = s.t["q"][torch.as_tensor(rows).cuda()].contiguous()
        want = torch.full((len(rows), s.nq, s.d), 7.0, dtype=s.out.dtype, device="cuda")
        call = lambda out, stream, q=q, where=where: s.pool.paged_prefix_attention8(q, out, s.t["ks"], s.t["vs"], *where, n_q_heads=s.nq,
                                                                                     stream=stream)
        call(want, None)
        torch.cuda.synchronize()
        s.out[torch.as_tensor(rows).cuda()] = want
        calls.append((call, want))
    s.check(lambda i: so.causal(*s.seqs[i]))
    return calls


@pytest.mark.parametrize("groups", [[[0, 1], [2, 3, 4]], [[0], [5]], [[0, 1, 3, 5], [2, 4]]], ids=str)
def test_two_streams_with_different_pieces(groups):
    """Partials of different queries, lengths and numbers of pieces at the same places of the workspace."""
    s = Setup("bf16", 8, 2, 128, LONG, kv8=True, seed=70).device()
    rest = [i for i in range(len(LONG)) if not any(i in g for g in groups)]
    calls = batches(s, groups + ([rest] if rest else []))[:2]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [(i % 2, torch.full_like(calls[i % 2][1], 3.0)) for i in range(32)]
    torch.cuda.synchronize()
    for which, out in outs:
        calls[which][0](out, streams[which])
    torch.cuda.synchronize()
    assert all(torch.equal(out, calls[which][1]) for which, out in outs)


def test_two_threads_with_different_lists():
    """Two threads, each with a stream and two kinds of calls: contexts that are cut, with the records staged, and lists of single tokens, staged
    as well; nobody waits before the end."""
    seqs = LONG + SHORT
    s = Setup("f16", 8, 2, 128, seqs, kv8=True, seed=71).device()
    a, b = list(range(6, 241)), list(range(241, 476))
    calls = batches(s, [[0, 1] + a, [2, 3, 4, 5] + b])
    calls += batches(s, [a + [0], b + [1, 2, 3, 4, 5]])
    failures, outs = [], [[], []]

    def run(mine):
        try:
            stream = torch.cuda.Stream()
            for i in range(40):
                which = mine + 2 * (i % 2)
                with torch.cuda.stream(stream):
                    out = torch.full_like(calls[which][1], 3.0)
                calls[which][0](out, stream)
                outs[mine].append((which, out))
            stream.synchronize()
        except Exception as e:                             # a thread's own would be lost
            failures.append(repr(e))

    torch.cuda.synchronize()
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failures
    assert all(torch.equal(out, calls[which][1]) for o in outs for which, out in o)
