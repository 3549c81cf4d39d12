"""The operators of a quantised cache and of drafted tokens as they are used together: the example, and a step in a graph."""
import os
import sys

import numpy as np
import pytest
import torch

import paper_2502_20969_amd as P
from quant import Problem8, verify

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_drafts_change_nothing_but_the_steps():
    """Token by token and with drafts, by itself and as a graph, the model says the same."""
    import answer_with_drafts as E
    texts, steps = E.answer(drafts=0, graph=False)
    assert steps == 39 and all(len(t) == 40 and min(t) >= 0 for t in texts)
    for kw in (dict(drafts=4), dict(drafts=4, graph=False), dict(drafts=1), dict(drafts=0)):
        again, n = E.answer(**kw)
        assert again == texts and n <= steps, kw


@pytest.mark.parametrize("seed", [0, 3, 5])
def test_drafts_save_steps(seed):
    """The model repeats itself: some of the drafts are what it says, more of four than of one, and its text stays the same.  (A verification that
    refused them all would take as many steps as tokens by themselves.)"""
    import answer_with_drafts as E
    (plain, steps), (one, n1), (four, n4) = (E.answer(drafts=d, seed=seed) for d in (0, 1, 4))
    assert one == plain and four == plain and n4 < n1 < steps == 39


def test_a_step_in_a_graph():
    """Append, attention, verification and reading back, captured once and replayed with other contents of the same tensors, eager work and waits
    between; two graphs with workspaces of their own in turn.  Every replay gives what the eager calls give."""
    vocab, hq = 700, 4
    pr = Problem8([3, 1, 5, 2], [40, 9, 300, 17], groups=[(3, 600)], hkv=2, d=64, dtype="f16", seed=3)
    step = pr.step(P, max_q=5, max_len=300, max_prefix=600)
    lens, start = step._keep[1], step._keep[1].clone()
    cache = pr.cache(P)
    g = torch.Generator().manual_seed(4)
    t = pr.tokens
    k, v = (torch.zeros(t, 2, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    q = torch.zeros(t, hq, 64, dtype=torch.float16, device="cuda")
    head = (torch.randn(hq * 64, vocab, generator=g) / 8).cuda()
    tokens, uniform = torch.zeros(t, dtype=torch.int32, device="cuda"), torch.zeros(t, device="cuda")
    draft = torch.zeros(t, vocab, device="cuda")
    off = torch.tensor([0, 640, 649, 949, 966], dtype=torch.int32).cuda()
    back = [torch.zeros(966, 2, 64, dtype=torch.float16, device="cuda") for _ in range(2)]
    logits = torch.zeros(t, vocab, device="cuda")

    def body():
        P.ivf_kv_append(step, cache, k, v)
        out = P.ivf_attend(step, cache, q)
        logits.copy_(out.view(t, -1).float() @ head)
        got = P.ivf_verify_draft(step, logits, tokens, uniform, draft=draft, lens_out=lens)
        P.ivf_kv_read(step, cache, off, *back)
        return [out, got[0], got[1], lens, *back]

    def fill(i):
        lens.copy_(start)
        for x, f in ((k, 1.0), (v, 2.0), (q, 1.0)):
            x.copy_(torch.randn(x.shape, generator=g) * f)
        tokens.copy_(torch.randint(0, vocab, (t,), generator=g))
        uniform.copy_(torch.rand(t, generator=g) * (0.002 if i % 2 else 1.0))
        draft.copy_(torch.softmax(torch.randn(t, vocab, generator=g), -1))

    fill(0)
    body()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        lens.copy_(start)
        one = torch.cuda.CUDAGraph()
        with torch.cuda.graph(one):
            res = body()
        graphs.append((one, res))
    seen = set()
    for i in range(6):
        fill(i)
        state = [x.clone() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale, *back)]
        want = [x.clone() for x in body()]
        torch.cuda.synchronize()
        for x, y in zip((cache.k, cache.v, cache.k_scale, cache.v_scale, *back), state):
            x.copy_(y)
        lens.copy_(start)
        graph, res = graphs[i % 2]
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(res, want):
            assert torch.equal(x, y)
        a, f, n, near = verify(logits.double().cpu().numpy(), tokens.cpu().numpy(), uniform.cpu().numpy(), np.asarray(pr.q_off), start.cpu().numpy(), draft.cpu().numpy())
        assert not near.any() and want[1].tolist() == a.tolist() and want[2].tolist() == f.tolist() and want[3].tolist() == n.tolist()
        seen |= set(want[1].tolist())
    assert len(seen) > 1


def test_calls_on_two_streams():
    """Two steps over caches of their own at once."""
    prs = [Problem8([1] * 6, [500 + 50 * i for i in range(6)], hkv=2, d=128, seed=s) for s in range(2)]
    streams = [torch.cuda.Stream() for _ in prs]
    qs = [pr.rows(8) for pr in prs]
    args = [(pr.step(P), pr.cache(P), q.cuda()) for pr, q in zip(prs, qs)]
    torch.cuda.synchronize()
    for _ in range(5):
        outs = [P.ivf_attend(*a, stream=s) for a, s in zip(args, streams)]
    torch.cuda.synchronize()
    for pr, q, out in zip(prs, qs, outs):
        want, _, tol = pr.attend(q, pr.d ** -0.5)
        assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
