"""The N-best lists of a transducer, rescored and continued by a transformer language model under the same beams.

    python examples/continue_nbest.py [--utts 8] [--beam 5] [--steps 20] [--together]

`tbs_decode` gives every utterance up to N token sequences.  A decoder-only transformer (random weights, as everything here is
synthetic) reads them token by token, all hypotheses of all utterances together, and then goes on under beam search.  One step of the model
is `linear` (products with bias, activation and residual) and `attend_paged` (one new token per hypothesis over its paged cache); one of
the search is `beam_select` and `beam_reorder`.  With --together the model reads all tokens of the lists in one pass instead: `page_slots` says where they
stand and go, `rotary` brings their keys and values into the cache and `attend_prompts` is their attention.  Token 0, the transducer's blank, ends a sequence.
"""

from __future__ import annotations

import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2302_14357_amd import attend_paged, attend_prompts, beam_reorder, beam_select, linear, page_slots, rotary  # noqa: E402

END = 0


class Lm:
    """Weights of a decoder-only transformer: `layers` blocks of attention (kv_heads key heads) and a feed-forward block, norms before each.  `turned`: queries and
    keys are turned by their positions, instead of a vector that is added for each."""

    def __init__(self, vocab, width=256, layers=2, heads=8, kv_heads=2, dtype=torch.bfloat16, seed=0, device="cuda", turned=False):
        g = torch.Generator().manual_seed(seed)
        self.heads, self.kv, self.dim, self.dtype, self.width, self.vocab = heads, kv_heads, width // heads, dtype, width, vocab

        def matrix(rows, cols, scale=1.0):
            return (torch.randn(rows, cols, generator=g) * scale / cols**0.5).to(dtype).to(device)

        def bias(n):
            return (0.05 * torch.randn(n, generator=g)).to(device)
        self.embed = (torch.randn(vocab, width, generator=g)).to(dtype).to(device)
        self.place = (torch.randn(4096, width, generator=g) * 0.3).to(dtype).to(device)
        self.blocks = [dict(qkv=matrix((heads + 2 * kv_heads) * self.dim, width), qkv_bias=bias((heads + 2 * kv_heads) * self.dim), out=matrix(width, width),
                            out_bias=bias(width), up=matrix(4 * width, width), up_bias=bias(4 * width), down=matrix(width, 4 * width), down_bias=bias(width))
                       for _ in range(layers)]
        self.head = matrix(vocab, width, 3.0)
        pairs = self.dim // 2 if turned else 0
        self.freqs = (10000.0 ** -(torch.arange(pairs, dtype=torch.float64) / max(pairs, 1))).to(device)
        self.turned = turned

    def enter(self, tokens, at):
        x = self.embed[tokens.long().clamp(min=0)]
        return x if self.turned else x + self.place[at]

    def heads_of(self, b, x):
        return linear(F.layer_norm(x, (self.width,)), b["qkv"], b["qkv_bias"]).view(len(x), -1, self.dim).split((self.heads, self.kv, self.kv), 1)

    def leave(self, b, x, o):
        x = linear(o.view(len(x), -1), b["out"], b["out_bias"], residual=x)
        h = linear(F.layer_norm(x, (self.width,)), b["up"], b["up_bias"], act="gelu")
        return linear(h, b["down"], b["down_bias"], residual=x)

    def logits(self, x):
        return linear(F.layer_norm(x, (self.width,)), self.head, out_dtype=torch.float32)


class Beams:
    """`rows` hypotheses, `beams` to an utterance, with room for max_len tokens each: their caches, page tables and lengths."""

    def __init__(self, lm, rows, beams, max_len, page=16):
        self.lm, self.beams, self.page = lm, beams, page
        width = -(-max_len // page)
        device = lm.embed.device
        self.tables = torch.arange(rows * width, dtype=torch.int32, device=device).view(rows, width)   # pages reserved ahead, none shared
        self.lens = torch.zeros(rows, dtype=torch.int32, device=device)
        self.caches = torch.empty(2 * len(lm.blocks), rows * width, page, lm.kv, lm.dim, dtype=lm.dtype, device=device)
        self.longest = 0

    def logits(self, tokens):
        """One token per hypothesis -> float32 logits of the next; hypotheses of negative length take no part."""
        lm = self.lm
        self.longest += 1
        at = self.lens.clamp(min=0)
        x = lm.enter(tokens, at.long())
        for i, b in enumerate(lm.blocks):
            q, k, v = lm.heads_of(b, x)
            if lm.turned:
                q, k = rotary(q, k, at, lm.freqs)
            o = attend_paged(q, self.caches[2 * i], self.caches[2 * i + 1], self.tables, self.lens, k_new=k, v_new=v, beams=self.beams, max_len=self.longest)
            x = lm.leave(b, x, o)
        return lm.logits(x)

    def read(self, tokens, count, longest):
        """All tokens of all hypotheses, one after the other, `count` int32 of each, up to `longest` -> float32 logits behind every token."""
        lm = self.lm
        self.longest = longest
        starts, at, slots = page_slots(count, self.tables, page=self.page, tokens=len(tokens))
        x = lm.enter(tokens, at.long())
        for i, b in enumerate(lm.blocks):
            q, k, v = lm.heads_of(b, x)
            q, k = rotary(q, k, at, lm.freqs, v=v, k_cache=self.caches[2 * i], v_cache=self.caches[2 * i + 1], slots=slots)
            x = lm.leave(b, x, attend_prompts(q, k, v, starts))
        return lm.logits(x)


@torch.no_grad()
def continue_nbest(lm, nbest, beams, steps, page=16, together=False):
    """nbest: per utterance up to `beams` (tokens, log score).  Returns the same after `steps` tokens more (fewer for those that end), best first, and how
    many hypotheses were dropped on the way (beam_reorder's status; they do not come back).  A score is the list's plus the model's logarithms of all tokens, the first one's behind END.
    `together`: the lists' tokens are read in one pass."""
    device = lm.embed.device
    rows = len(nbest) * beams
    said = [[END] + list(nb[i][0]) if i < len(nb) else [] for nb in nbest for i in range(beams)]
    scores = torch.tensor([nb[i][1] if i < len(nb) else -torch.inf for nb in nbest for i in range(beams)], dtype=torch.float64, device=device)
    length = max(len(s) for s in said)
    given = torch.full((rows, length), -1, dtype=torch.long)
    for r, s in enumerate(said):
        given[r, :len(s)] = torch.tensor(s)
    given, count = given.to(device), torch.tensor([len(s) for s in said], device=device)
    state = Beams(lm, rows, beams, length + steps, page)
    last = torch.empty(rows, lm.vocab, dtype=torch.float32, device=device)
    if together and length > 0:   # (lists may all be empty)
        flat = torch.tensor([t for s in said for t in s], device=device)
        logits = state.read(flat, count.int(), length)
        last = logits[(count.cumsum(0) - 1).clamp(min=0)]
        # what the model says of every hypothesis' next tokens, a row of its own for each
        here = torch.arange(length, device=device) < count[:, None]
        said_next = torch.zeros(rows, length, dtype=torch.float64, device=device)
        said_next[here] = torch.log_softmax(logits.double(), 1).gather(1, flat.roll(-1)[:, None])[:, 0]
        scores = scores + said_next.masked_fill(torch.arange(length, device=device) >= count[:, None] - 1, 0.0).sum(1)
    for t in range(0 if together else length):
        here = t < count
        state.lens = torch.where(here, t, ~(count.clamp(max=t))).int()
        logits = state.logits(given[:, t])
        last = torch.where(here[:, None], logits, last)
        if t + 1 < length:   # what the model says of the next token that is given
            said_next = torch.log_softmax(logits.double(), 1).gather(1, given[:, t + 1].clamp(min=0)[:, None])[:, 0]
            scores = scores + torch.where(t + 1 < count, said_next, 0.0)
    state.lens = torch.where(count > 0, count - 1, -1).int()   # (the last given token is the first step's)
    done = torch.zeros(rows, dtype=torch.bool, device=device)
    logits, dropped, path = last, torch.zeros(1, dtype=torch.int32, device=device), []
    for t in range(steps):
        scores, tokens, parents, done = beam_select(logits, scores, beams=beams, finished=done, eos=END)
        path.append((tokens, parents))
        if t + 1 < steps:
            state.tables, state.lens = beam_reorder(parents, state.tables, state.lens, state.caches, beams=beams, finished=done, status=dropped)
            scores = scores.masked_fill((state.lens == -1) & ~done, -torch.inf)   # a hypothesis that was dropped has no tokens to go on from
            logits = state.logits(tokens)
    # the sequences, from the last step back
    path = [(t.view(-1, beams).tolist(), p.view(-1, beams).tolist()) for t, p in path]
    out = []
    for u, row in enumerate(scores.view(-1, beams).tolist()):
        mine = []
        for i, s in enumerate(row):
            if s == -torch.inf:
                continue
            tail, at = [], i
            for tokens, parents in reversed(path):
                tail.append(tokens[u][at])
                at = parents[u][at]
            tail = tail[::-1]
            if END in tail:
                tail = tail[:tail.index(END) + 1]   # (a sequence that has ended repeats its end)
            mine.append((tuple(said[u * beams + at][1:] + tail), s))
        out.append(mine)
    return out, int(dropped)


def main():
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--utts", type=int, default=8)
    a.add_argument("--beam", type=int, default=5)
    a.add_argument("--steps", type=int, default=20)
    a.add_argument("--together", action="store_true")
    a = a.parse_args()
    import dataclasses
    from paper_2302_14357_amd import Tbs
    from tbs_inputs import SHAPES, make_model, make_utterances
    shape = dataclasses.replace(SHAPES["librispeech"], n_utts=a.utts, len_lo=20, len_hi=60, logit_scale=8.0, blank_bias=8.0)   # peaked: sequences of several tokens
    model = make_model(shape)
    offsets, enc = make_utterances(shape, model)
    tbs = Tbs(model, blank_id=shape.blank_id, beam_n=a.beam, seg_s=3, max_utts=a.utts, max_frames_total=int(offsets[-1]), dtype="bf16", act=shape.act,
              max_rounds_per_segment=6)
    nbest = tbs.decode(tbs.upload_frames(enc), offsets)
    tbs.close()
    got, dropped = continue_nbest(Lm(shape.vocab), nbest, a.beam, a.steps, together=a.together)
    for u, (before, after) in enumerate(zip(nbest, got)):
        print(f"utterance {u}: {len(before)} hypotheses of {min(len(t) for t, _ in before)} to {max(len(t) for t, _ in before)} tokens; now best: "
              f"{list(after[0][0])} ({after[0][1]:.3f})")
    print("hypotheses dropped:", dropped)


if __name__ == "__main__":
    main()
