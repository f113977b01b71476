"""The operators together, as examples/continue_nbest.py uses them, against the same model in float64 without a cache."""

import os
import sys

import pytest
import torch
import torch.nn.functional as F

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _plain_logits(lm, tokens):
    """Logits behind every prefix of `tokens`, float64 on the CPU."""
    d = lambda t: t.detach().cpu().double()   # noqa: E731
    n, g = len(tokens), lm.heads // lm.kv
    x = d(lm.embed)[tokens] + d(lm.place)[:n]
    mask = torch.full((n, n), float("-inf"), dtype=torch.float64).triu(1)
    for b in lm.blocks:
        qkv = (F.layer_norm(x, (lm.width,)) @ d(b["qkv"]).T + d(b["qkv_bias"])).view(n, -1, lm.dim)
        q, k, v = qkv.split((lm.heads, lm.kv, lm.kv), 1)
        k, v = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
        p = torch.softmax(torch.einsum("ihd,jhd->hij", q, k) / lm.dim**0.5 + mask, -1)
        x = x + torch.einsum("hij,jhd->ihd", p, v).reshape(n, -1) @ d(b["out"]).T + d(b["out_bias"])
        h = F.layer_norm(x, (lm.width,)) @ d(b["up"]).T + d(b["up_bias"])
        x = x + (h * torch.special.ndtr(h)) @ d(b["down"]).T + d(b["down_bias"])
    return F.layer_norm(x, (lm.width,)) @ d(lm.head).T


def _plain_score(lm, start, tokens):
    l = torch.log_softmax(_plain_logits(lm, [0] + list(tokens[:-1])), 1) if tokens else None
    return start + (sum(float(l[i, t]) for i, t in enumerate(tokens)) if tokens else 0.0)


def _plain_beam(lm, nbest, beams, steps):
    """The search itself, over whole sequences, and the smallest gap of a decision it took."""
    alive, gap = [(tuple(t), _plain_score(lm, s, t), False) for t, s in nbest], float("inf")
    for _ in range(steps):
        cand = []
        for i, (t, s, done) in enumerate(alive):
            if done:
                cand.append((s, i, t, True))
                continue
            l = torch.log_softmax(_plain_logits(lm, [0] + list(t))[-1], 0)
            top = torch.topk(l, beams + 1)
            cand += [(s + float(x), i, t + (int(v),), int(v) == 0) for x, v in zip(top.values, top.indices)]
        cand.sort(key=lambda c: (-c[0], c[1]))
        if len(cand) > beams:
            gap = min([gap] + [cand[j][0] - cand[j + 1][0] for j in range(beams)])
        alive = [(t, s, done) for s, _, t, done in cand[:beams]]
    return [(t, s) for t, s, _ in alive], gap


# A float32 model's logits are off by some float32 units of the sums they come from: below 1e-5 each here, 40 tokens' logarithms below 1e-3
TOL = 1e-3


@pytest.mark.parametrize("page", [4, 16])
def test_continue_nbest_float32(page):
    from continue_nbest import Lm, continue_nbest
    lm = Lm(60, width=64, layers=2, heads=4, kv_heads=2, dtype=torch.float32, seed=page)
    g = torch.Generator().manual_seed(5)
    nbest = []
    for u in range(6):   # lists of different lengths, hypotheses of 0 to 13 tokens, an utterance with one hypothesis and one with an empty one
        n = [4, 1, 3, 2, 4, 4][u]
        nbest.append([(tuple(torch.randint(1, 60, (int(torch.randint(0, 14, (1,), generator=g)),), generator=g).tolist()), -float(i) - u) for i in range(n)])
    got, dropped = continue_nbest(lm, nbest, 4, 12, page=page)
    assert dropped == 0
    clear = 0
    for mine, start in zip(got, nbest):
        want, gap = _plain_beam(lm, start, 4, 12)
        for t, s in mine:   # every returned sequence has the score that it has in float64
            base = [p for p, _ in start if t[:len(p)] == p]
            assert base
            assert min(abs(s - _plain_score(lm, b, t)) for p, b in start if t[:len(p)] == p) < TOL
        assert all(a[1] >= b[1] for a, b in zip(mine, mine[1:]))
        if gap > 2 * TOL:   # every decision was clear: the same sequences in the same order
            clear += 1
            assert [t for t, _ in mine] == [t for t, _ in want]
    assert clear >= 2


def test_continue_nbest_with_dropped_hypotheses():
    """Lists of very different lengths and about equal scores, pages of one token: some hypotheses have to be dropped, and none of theirs comes back with a score
    that is not its own."""
    from continue_nbest import Lm, continue_nbest
    lm = Lm(40, width=64, layers=1, heads=4, kv_heads=2, dtype=torch.float32, seed=3)
    g = torch.Generator().manual_seed(8)
    nbest = []
    for u in range(8):
        lists = [tuple(torch.randint(1, 40, (n,), generator=g).tolist()) for n in (0, 3, 9, 14)]
        nbest.append([(t, -_plain_score(lm, 0.0, t) - 3.0 * float(torch.rand(1, generator=g))) for t in lists])
    got, dropped = continue_nbest(lm, nbest, 4, 10, page=1)
    assert dropped > 0
    for mine, start in zip(got, nbest):
        assert mine and all(a[1] >= b[1] for a, b in zip(mine, mine[1:]))
        for t, s in mine:
            assert min(abs(s - _plain_score(lm, b, t)) for p, b in start if t[:len(p)] == p) < TOL


def test_example_runs_on_the_transducers_lists(capsys, monkeypatch):
    import continue_nbest
    monkeypatch.setattr(sys, "argv", ["continue_nbest.py", "--utts", "3", "--beam", "4", "--steps", "6"])
    continue_nbest.main()
    out = capsys.readouterr().out
    assert out.count("utterance ") == 3 and "hypotheses dropped: 0" in out
