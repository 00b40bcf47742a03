"""Greedy decoding over a closed set of strings, several tokens per step: the set's own continuations are drafted as a tree, one
step of the model looks at all of them, and the path that it confirms stays in the cache.

    python examples/drafts.py

A step: draft a tree below the last token (the longest tokens that the set allows, level by level), make room for it, append
the layer's K, V and turned queries, attend through the tree's mask, mask the logits by the tokens' trie nodes, pick the best
token after each, keep the path that the picks follow.  The strings are those that one token per step finds.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch
import torch.nn.functional as F

import paper_2608_12574_amd as tam
from examples import beams


class Decoder(beams.Decoder):
    """The beams' decoder with positions: queries and keys turn by them."""

    def __init__(self, vocab, head_dim=64, base=10000.0, **kw):
        super().__init__(vocab, head_dim=head_dim, **kw)
        self.frequencies = base ** -(torch.arange(0, head_dim, 2, device="cuda", dtype=torch.float32) / head_dim)

    def __call__(self, tokens, cache, slots, offsets=None, longest=None, depth=None, seen=None):
        """[tokens, vocab] logits of the slots' last tokens, which the cache has room for (``extend``): a run of text each, or
        trees (``depth`` and ``seen``, see ``tree_masks``)."""
        x = self.embed[tokens.long().clamp(min=0)]
        norm = lambda x: F.rms_norm(x, x.shape[-1:])
        q_width, kv_width = self.heads * self.head_dim, self.kv_heads * self.head_dim
        rows = dict(offsets=offsets, slots=slots, longest=longest)
        for i, (qkv, out, up, down) in enumerate(self.layers):
            q, k, v = F.linear(norm(x), qkv).split([q_width, kv_width, kv_width], 1)
            k, v = (t.unflatten(1, (self.kv_heads, self.head_dim)) for t in (k, v))
            q = cache.append(i, q.unflatten(1, (self.heads, self.head_dim)), k, v, self.frequencies, depth=depth, **rows)
            y = cache.attend(i, q, seen=seen, **rows)
            x = x + F.linear(y.flatten(1), out)
            gate, y = F.linear(norm(x), up).chunk(2, 1)
            x = x + F.linear(F.silu(gate) * y, down)
        return F.linear(norm(x), self.head)


def shape(levels):
    """Parents of a tree whose tokens have levels[d] children at depth d, depth by depth."""
    parents, last = [-1], [0]
    for n in levels:
        first = len(parents)
        parents += [p for p in last for _ in range(n)]
        last = range(first, len(parents))
    return parents


def generate(model, handle, prior, prompts, levels=(4, 2, 1), most=32, page_tokens=16):
    """The greedy continuation of each prompt, the steps that it took and the cache: (tokens, steps, cache).  ``prior`` [V]: what is
    drafted first; no ``levels``: one token per step; ``most``: steps at most, each of which adds up to len(levels) + 1 tokens."""
    B, V = len(prompts), len(prior)
    int32 = dict(dtype=torch.int32, device="cuda")
    begin = [len(p) for p in prompts]
    parents = shape(levels)
    n = len(parents)
    held = -(-(max(begin) + most * (len(levels) + 1) + n) // page_tokens)  # what stays, and a tree behind it
    cache = tam.PageCache.empty(len(model.layers), model.kv_heads, model.head_dim, pages=B * held, slots=B, max_pages=held,
                                page_tokens=page_tokens)
    slots = torch.arange(B, **int32)

    # the prompts, and the first token after each
    cache.extend(slots, torch.tensor(begin, **int32))
    offsets = torch.tensor([sum(begin[:i]) for i in range(B + 1)], **int32)
    logits = model(torch.tensor(sum(prompts, []), **int32), cache, slots, offsets, max(begin))[(offsets[1:] - 1).long()]
    nodes = torch.zeros(B, **int32)
    handle.adjust_logits(nodes, logits)
    token = tam.top_tokens(logits, 1)[0].view(B)
    nodes = handle.advance(nodes, token)
    text, steps = [[t] for t in token.tolist()], 0

    # every tree has the same shape, so its masks are made once
    up = torch.tensor(parents * B, **int32)
    offsets = torch.arange(0, B * n + 1, n, **int32)
    seen, depth = tam.tree_masks(up, offsets, longest=n)
    counts = torch.full((B,), n, **int32)
    alive = torch.ones(B, dtype=torch.bool, device="cuda")
    while steps < most:
        # level by level; where the set allows fewer children than there is room for, token -1 at node -1 is no one's choice
        tree, at = [token.view(B, 1)], [nodes.view(B, 1)]
        for k in levels:
            weights = prior.repeat(at[-1].numel(), 1)
            handle.apply_mask(at[-1].reshape(-1), weights)
            best = tam.top_tokens(weights, k)[0].view(B, -1)
            then = handle.advance(at[-1].repeat_interleave(k, 1).reshape(-1), best.reshape(-1)).view(B, -1)
            tree.append(best)
            at.append(torch.where(best < 0, -1, then))
        tree, at = torch.cat(tree, 1).reshape(-1), torch.cat(at, 1).reshape(-1).contiguous()

        cache.extend(slots, torch.where(alive, counts, 0))
        logits = model(tree, cache, slots, offsets, n, depth, seen)
        handle.adjust_logits(at, logits)
        picks = tam.top_tokens(logits, 1)[0].view(-1)
        path, count, last = cache.accept(tree, picks, up, offsets=offsets, slots=slots)
        steps += 1

        # the last token that stays, its node, and the choice after it (-1 where the string is over)
        end = (path.view(B, n).gather(1, (count.long() - 1)[:, None]) + offsets[:-1, None])[:, 0].long()
        nodes = handle.advance(at[end], last)
        token = last
        for b, (p, c, t) in enumerate(zip(path.view(B, n).tolist(), count.tolist(), last.tolist())):
            if text[b][-1] >= 0:
                text[b] += tree.view(B, n)[b, p[1:c]].tolist() + [t]
        alive = alive & (last >= 0)
        if not bool(alive.any()):
            break
        # strings that are over leave their slots empty
        slots_over = torch.where(alive, slots, -1)
        cache.fork(slots, slots_over)
    cache.free(slots)
    return [t[:-1] if t[-1] < 0 else t for t in text], steps, cache


def main():
    vocab = beams.vocabulary()
    handle = tam.compile(beams.STRINGS, vocab, device="cuda:0")
    prior = torch.tensor([float(len(t)) for t in vocab], device="cuda")
    prompts = [list(b"Which fruit is it?"), list(b"And the other one, which lay beside it: ")]
    model = Decoder(len(vocab))
    for levels in ((), (4, 2, 1)):
        found, steps, _ = generate(model, handle, prior, prompts, levels)
        print("%d tokens per step of each string, %d steps" % (len(shape(levels)), steps))
        for prompt, tokens in zip(prompts, found):
            print("  %s -> %s" % (bytes(prompt).decode(), b"".join(vocab[t] for t in tokens)[:-1].decode()))


if __name__ == "__main__":
    main()
