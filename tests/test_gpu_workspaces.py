"""GPU tests of the workspaces that the binding hands to the calls on logits: one for each call, so that neither threads on one stream
nor captured graphs meet in one, and a status word stays its call's."""
import threading

import pytest
import torch

from paper_2512_16273_b200 import synth, tslt

pytestmark = pytest.mark.gpu


def case(seed, B=6, gamma=3, V=20000, k=32):
    zq, zp = synth.sequence_logits(B, gamma, V, torch.bfloat16, 0.5, seed, "cpu")
    u = {"d": synth.uniforms((B * gamma, 1), seed, synth.TID_U_DRAFT), "a": synth.uniforms((B, gamma), seed, synth.TID_U_ACCEPT),
         "s": synth.uniforms((B,), seed, synth.TID_U_SAMPLE)}
    return zq.cuda(), zp.cuda(), {n: t.cuda() for n, t in u.items()}, (B, gamma, V, k)


def run(c):
    zq, zp, u, (B, gamma, V, k) = c
    s = tslt.sparsify(zq.reshape(-1, V), k, 1.0, 0.9, u["d"])
    d = (s["idx"].view(B, gamma, k), s["logit"].view(B, gamma, k), s["count"].view(B, gamma), s["token"].view(B, gamma))
    return s, tslt.verify(zp, *d, 0.9, 0.9, u["a"], u["s"])


def tokens(pair):
    return [pair[0][n] for n in ("idx", "count", "token")] + [pair[1][n] for n in ("accepted_len", "out_token")]


def test_a_workspace_for_each_call():
    c = case(1)
    outs = [o for _ in range(2) for o in run(c)]
    assert len({o["workspace"].data_ptr() for o in outs}) == len(outs)
    assert [tslt.workspace_status(o["workspace"]) for o in outs] == [0] * len(outs)


def test_a_captured_call_has_its_own():
    """An ordinary call before the capture, and a larger one after it, use other memory than the graph."""
    c = case(2)
    want = [t.clone() for t in tokens(run(c))]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pair = run(c)
    held = {o["workspace"].data_ptr() for o in pair}
    later = run(case(3, B=40, V=30000))
    assert held.isdisjoint(o["workspace"].data_ptr() for o in later)
    for o in later:
        o["workspace"].fill_(255)  # and nothing of the graph's is in it
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(tokens(pair), want))


def test_threads_on_one_stream():
    cases = [case(10 + i, V=20000 + 512 * i) for i in range(4)]
    want = [[t.clone() for t in tokens(run(c))] for c in cases]
    torch.cuda.synchronize()
    got = [[] for _ in cases]
    start = threading.Barrier(len(cases))

    def work(i):
        start.wait()
        for _ in range(30):
            got[i].append(tokens(run(cases[i])))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(cases))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert len(a) == 30 and all(torch.equal(x, y) for o in a for x, y in zip(o, b))
