"""A chat within a budget, drafted in trees, with the one-layer model of speculative.py.

    python examples/long_chat.py [--steps 24] [--budget 448] [--batch 3]

Per step, for every sequence: the draft model proposes a tree (the last token, a few children,
and a child of each); the target runs over all its rows in one optr_tree_attention_win;
optr_verify_tree accepts a way down and draws the next token; optr_kv_append_win writes the
way's rows, and optr_kv_score_win adds the weights that they give to the cached positions.
A cache past its budget keeps the first, the recent and the most attended positions
(optr_evict_select, optr_kv_compact_win) and goes on behind them.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from speculative import CONFIG, D, H, VOCAB, Cache, Model, check, ints, offsets, optr  # noqa: E402


class Chat(Cache):
    """The cache and its account of attention."""

    def __init__(self, B, max_len, seed):
        super().__init__(B, max_len, seed)
        self.score = torch.zeros(B, H, 16 * self.table.shape[1], device="cuda")

    def attend_tree(self, q, k, v, parent, rows):
        out = torch.empty_like(q)
        B = len(self.len)
        ws = optr.new_chunk_workspace(self.p, q.shape[0], B, rows)
        optr.optr_tree_attention_win(self.p, q, k, v, parent, offsets([rows] * B), ints(self.len), rows,
                                     self.table, self.pool, self.win, self.slots, out, ws)
        return out

    def count(self, q, lens):
        """The weights that the last lens[b] cached tokens (their queries q) give."""
        B, most = len(lens), max(lens)
        ws = optr.new_score_workspace(self.p, q.shape[0], B, most, self.table.shape[1])
        optr.optr_kv_score_win(self.p, q, offsets(lens), ints([n - m for n, m in zip(self.len, lens)]), most,
                               self.table, self.pool, self.win, self.slots, self.score, ws)

    def shrink(self, budget):
        B = len(self.len)
        most = max(budget, CONFIG["sink"] + CONFIG["recent"])
        kept = torch.empty(B, H, most, dtype=torch.int32, device="cuda")
        n, n_kept = ints(self.len), torch.empty(B, dtype=torch.int32, device="cuda")
        optr.optr_evict_select(self.p, self.score, n, ints([budget] * B), CONFIG["sink"], CONFIG["recent"], kept,
                               n_kept)
        optr.optr_kv_compact_win(self.p, kept, n_kept, n, self.table, self.pool, self.win, self.slots, self.score)
        self.len = n_kept.tolist()


def step(model, chat, last, width, g):
    """Draft a tree, check it, keep a way of it: the new tokens of each sequence."""
    B, rows = len(last), 1 + 2 * width
    parent = [-1] + [0] * width + list(range(1, width + 1))
    q0 = model.probs(model.emb[last])
    first = torch.multinomial(q0, width, replacement=True, generator=g)           # drawn independently
    q1 = model.probs(model.emb[first.flatten()])
    second = torch.multinomial(q1, 1, generator=g).view(B, width)
    tokens = torch.cat((last[:, None], first, second), 1)
    q = torch.cat((q0[:, None], q1.view(B, width, VOCAB), torch.zeros(B, width, VOCAB, device="cuda")), 1)
    x = model.emb[tokens.flatten()]
    qh, k, v = model.qkv(x)
    tree = ints(parent * B)
    p = model.probs(x, chat.attend_tree(qh, k, v, tree, rows))
    accepted = torch.empty(B, dtype=torch.int32, device="cuda")
    path, out = (torch.empty(B * rows, dtype=torch.int32, device="cuda") for _ in range(2))
    noise = torch.empty(B, VOCAB, device="cuda").exponential_(generator=g).clamp_(min=1e-30)
    optr.optr_verify_tree(chat.p, p, q.view(-1, VOCAB), tokens.flatten().int(), tree,
                          torch.rand(B * rows, device="cuda", generator=g), noise, offsets([rows] * B), accepted,
                          path, out)
    keep = [a + 1 for a in accepted.tolist()]  # the last token and the accepted drafts
    at = torch.cat([path[b * rows:b * rows + n] for b, n in enumerate(keep)]).long()
    chat.write(k[at], v[at], keep)
    chat.count(qh[at], keep)
    return [r[:n].tolist() for r, n in zip(out.view(B, -1), keep)]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=24)
    ap.add_argument("--width", type=int, default=3)
    ap.add_argument("--batch", type=int, default=3)
    ap.add_argument("--prompt", type=int, default=430)
    ap.add_argument("--budget", type=int, default=448)
    a = ap.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(0)
    model = Model(1)
    prompts = [a.prompt + 37 * b for b in range(a.batch)]
    room = a.budget + 32
    chat = Chat(a.batch, max(room, max(prompts)) + 3, seed=2)
    text = [torch.randint(VOCAB, (n,), device="cuda", generator=g).tolist() for n in prompts]
    part = [t[:-1] for t in text]
    qh, k, v = model.qkv(model.emb[torch.tensor(sum(part, []), device="cuda")])
    chat.write(k, v, [len(t) for t in part])  # one layer: the prompt's rows are kept, its
    chat.count(qh, [len(t) for t in part])    # tokens' weights counted
    made = shrunk = 0
    for _ in range(a.steps):
        if max(chat.len) + 3 > room:
            chat.shrink(a.budget)
            shrunk += 1
        new = step(model, chat, torch.tensor([t[-1] for t in text], device="cuda"), a.width, g)
        for t, n in zip(text, new):
            t += n
            made += len(n)
    check(chat)
    print(f"{made} tokens in {a.steps} steps of {a.batch} sequences, {made / (a.steps * a.batch):.2f} a step; "
          f"the caches cut {shrunk} times to {a.budget}")
    return text, chat, made, shrunk


if __name__ == "__main__":
    main()
