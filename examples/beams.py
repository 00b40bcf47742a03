"""Beam search over a closed set of strings: a small decoder with random weights, whose every step runs the
library's operators as a serving loop would.

    python examples/beams.py

A step: fork the cache from the surviving beams, make room for one token each, store the layer's new K and V, attend,
adjust the logits (penalties, and the mask of the beams' trie nodes), pick the best continuations, advance
the nodes.  The prompt runs through the same calls as one chunk.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch
import torch.nn.functional as F

import paper_2608_12574_amd as tam


class Decoder:
    """Pre-norm attention and a gated layer, bf16, without positions; K and V live in a PageCache."""

    def __init__(self, vocab, layers=2, heads=8, kv_heads=2, head_dim=64, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        width = heads * head_dim

        def weight(n_out, n_in):
            return (torch.randn((n_out, n_in), generator=g, device="cuda") / n_in ** 0.5).to(torch.bfloat16)
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.embed = weight(vocab, width) * width ** 0.5
        self.layers = [(weight(width + 2 * kv_heads * head_dim, width), weight(width, width), weight(4 * width, width),
                        weight(width, 2 * width)) for _ in range(layers)]
        self.head = weight(vocab, width)

    def __call__(self, tokens, cache, slots, offsets=None, longest=None):
        """[tokens, vocab] logits of the slots' last tokens; the cache has room for them (``extend``)."""
        x = self.embed[tokens.long()]
        norm = lambda x: F.rms_norm(x, x.shape[-1:])
        q_width, kv_width = self.heads * self.head_dim, self.kv_heads * self.head_dim
        for i, (qkv, out, up, down) in enumerate(self.layers):
            q, k, v = F.linear(norm(x), qkv).split([q_width, kv_width, kv_width], 1)
            k, v = (t.unflatten(1, (self.kv_heads, self.head_dim)) for t in (k, v))
            cache.store(i, k, v, offsets=offsets, slots=slots, longest=longest)
            y = cache.attend(i, q.unflatten(1, (self.heads, self.head_dim)), offsets=offsets, slots=slots, longest=longest)
            x = x + F.linear(y.flatten(1), out)
            gate, y = F.linear(norm(x), up).chunk(2, 1)
            x = x + F.linear(F.silu(gate) * y, down)
        return F.linear(norm(x), self.head)


def search(model, handle, ends, prompts, width=4, most=32, presence=0.3, page_tokens=16):
    """The finished beams of each prompt, best first: [(score, tokens after the prompt)].  ``ends`` [V]: whether a
    token closes its string; ``width``: beams of each prompt, up to the 64 tokens that ``top_tokens`` gives."""
    groups = len(prompts)
    B = groups * width
    int32 = dict(dtype=torch.int32, device="cuda")
    longest = max(len(p) for p in prompts)
    held = -(-(longest + most) // page_tokens)
    cache = tam.PageCache.empty(len(model.layers), model.kv_heads, model.head_dim, pages=B * (held + 1), slots=B,
                                max_pages=held, page_tokens=page_tokens)
    text = torch.zeros((B, longest + most), **int32)  # each beam's tokens
    for i, p in enumerate(prompts):
        text[i * width:(i + 1) * width, :len(p)] = torch.tensor(p, **int32)
    begin = torch.tensor([len(p) for p in prompts], **int32).repeat_interleave(width)
    penalty = torch.full((B,), presence, device="cuda")

    # the prompts: a chunk in the first slot of each group
    first, slots = torch.arange(0, B, width, **int32), torch.arange(B, **int32)
    cache.extend(first, begin[::width].contiguous())
    offsets = F.pad(begin[::width].cumsum(0), (1, 0)).to(torch.int32)
    logits = model(torch.tensor(sum(prompts, []), **int32), cache, first, offsets, longest)
    logits = logits[(offsets[1:] - 1).long()].repeat_interleave(width, 0)

    score = torch.full((groups, width), -torch.inf, device="cuda")
    score[:, 0] = 0
    nodes = torch.zeros(B, **int32)
    ones = torch.ones(B, **int32)
    done = [[] for _ in prompts]
    for step in range(most):
        at = begin + step
        handle.adjust_logits(nodes, logits, tokens=text, length=at, prompt=begin, presence=penalty)
        # a group's best continuations are among each beam's (of a dead beam: token -1 at -inf)
        best, total = tam.top_tokens(logits, width)
        score, pick = (total + score.view(B, 1)).view(groups, width * width).topk(width, 1)
        parents = (pick // width + torch.arange(0, B, width, device="cuda")[:, None]).view(B).to(torch.int32)
        token = best.view(groups, width * width).gather(1, pick).view(B)
        text = text[parents.long()]
        text[slots.long(), at.long()] = token
        nodes = handle.advance(nodes[parents.long()], token)
        alive = score.view(B) > -torch.inf
        over = alive & ends[token.long()]
        for b in over.nonzero().flatten().tolist():
            done[b // width].append((float(score.view(B)[b]), text[b, int(begin[b]):int(at[b]) + 1].tolist()))
        alive &= ~over
        score = torch.where(alive.view(groups, width), score, -torch.inf)
        if not bool(alive.any()):
            break
        # beams that end give their pages back
        cache.fork(slots, torch.where(alive, parents, -1))
        cache.extend(slots, torch.where(alive, ones, 0))
        logits = model(token, cache, slots)
    cache.free(slots)
    return [sorted(d, key=lambda x: -x[0]) for d in done], cache


def vocabulary():
    """Every byte, and some longer tokens."""
    return [bytes([b]) for b in range(256)] + [b"red", b"green", b"blue", b" app", b"le", b"grape", b" p", b"ear", b's"']


STRINGS = [b"red apple", b"red apples", b"green apple", b"green pear", b"blue grapes", b"blue grape", b"red grapes"]


def main():
    vocab = vocabulary()
    handle = tam.compile(STRINGS, vocab, device="cuda:0")
    ends = torch.tensor([t.endswith(b'"') for t in vocab], device="cuda")
    prompts = [list(b"Which fruit is it?"), list(b"And the other one, which lay beside it: ")]
    found, _ = search(Decoder(len(vocab)), handle, ends, prompts)
    for prompt, beams in zip(prompts, found):
        print(bytes(prompt).decode())
        for score, tokens in beams:
            print("  %7.3f  %s" % (score, b"".join(vocab[t] for t in tokens)[:-1].decode()))


if __name__ == "__main__":
    main()
