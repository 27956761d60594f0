"""Speculative decoding over the INT2 cache, with a one-layer model of random
weights: the prompt in chunks, then per step a few drafted tokens checked at
once, and at the end the cache moved to other rotations.

    python examples/speculative.py [--steps 24] [--drafts 4] [--batch 3]

Per step, for every sequence: the draft model (the same model without its
attention) proposes tokens; the target runs over the last token and the drafts
in one optr_chunk_attention_win, which reads the cache and leaves it alone;
optr_verify_drafts accepts a prefix and draws the next token, so the text has
the target's distribution; optr_kv_append_win writes the rows that stay.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_02691_gb300 import optr, synth  # noqa: E402

H, D, WIDTH, VOCAB = 2, optr.HEAD_DIM, 512, 4001
CONFIG = dict(group=128, clip_k=0.96, clip_v=0.92, sink=64, recent=256)


class Model:
    """x -> x + attention(x) -> probabilities; without attention, the draft."""

    def __init__(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda *s: (torch.randn(*s, device="cuda", generator=g) * s[0] ** -0.5).bfloat16()
        self.emb = VOCAB ** 0.5 * w(VOCAB, WIDTH)
        self.wq, self.wk, self.wv = w(WIDTH, 4 * H * D), w(WIDTH, H * D), w(WIDTH, H * D)
        self.wo, self.head = 2 * w(4 * H * D, WIDTH), 3 * w(WIDTH, VOCAB)

    def qkv(self, x):
        return tuple((x @ w).view(x.shape[0], -1, D) for w in (self.wq, self.wk, self.wv))

    def probs(self, x, attn=None):
        if attn is not None:
            x = x + attn.reshape(x.shape[0], -1) @ self.wo
        return torch.softmax((x @ self.head).float(), 1)


class Cache:
    """One layer's pages and windows for B sequences of at most max_len tokens."""

    def __init__(self, B, max_len, seed):
        R_k, R_v = synth.rotations(H, seed)
        self.p = optr.optr_params_create(R_k, R_v, torch.zeros(H, D), 4 * H, **CONFIG)
        pages = -(-max_len // 16)  # tokens of a page
        self.pool = optr.new_pool(self.p, B * pages)
        self.table = torch.randperm(B * pages).view(B, pages).int().cuda()
        self.win, self.slots = optr.new_windows(self.p, B), torch.arange(B, dtype=torch.int32).cuda()
        self.len = [0] * B

    def attend(self, q, k, v, lens):
        """The new tokens, lens[b] of each sequence, over the cache and themselves."""
        out = torch.empty_like(q)
        ws = optr.new_chunk_workspace(self.p, q.shape[0], len(lens), max(lens))
        optr.optr_chunk_attention_win(self.p, q, k, v, offsets(lens), ints(self.len), max(lens), self.table,
                                      self.pool, self.win, self.slots, out, ws)
        return out

    def write(self, k, v, lens):
        optr.optr_kv_append_win(self.p, k, v, offsets(lens), ints(self.len), self.table, self.pool, self.win,
                                self.slots)
        self.len = [a + b for a, b in zip(self.len, lens)]

    def rows(self):
        """Every sequence's cached keys and values, as one batch."""
        k = torch.empty(sum(self.len), H, D, dtype=torch.bfloat16, device="cuda")
        v = torch.empty_like(k)
        optr.optr_kv_read(self.p, offsets(self.len), ints([0] * len(self.len)), self.table, self.pool, k, v)
        r0 = 0
        for b, n in enumerate(self.len):  # the windows hold their rows exactly
            pos = torch.arange(n, device="cuda")
            for lo, hi, at in ((0, min(n, CONFIG["sink"]), pos),
                               (max(CONFIG["sink"], n - CONFIG["recent"]), n,
                                CONFIG["sink"] + (pos - CONFIG["sink"]) % CONFIG["recent"])):
                if lo < hi:
                    kv = self.win[int(self.slots[b])][:, :, at[lo:hi]]  # [H][2][rows][D]
                    k[r0 + lo:r0 + hi], v[r0 + lo:r0 + hi] = kv[:, 0].transpose(0, 1), kv[:, 1].transpose(0, 1)
            r0 += n
        return k, v


def check(cache):
    flags = optr.optr_device_error(cache.p)
    if flags:
        raise RuntimeError(f"device error flags {flags}")


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def offsets(lens):
    return torch.nn.functional.pad(ints(lens).cumsum(0, dtype=torch.int32), (1, 0))


def step(model, cache, last, n_draft, g):
    """Draft, check and keep: the new tokens of each sequence."""
    B = len(last)
    x, tokens, q = model.emb[last], [last], []
    for _ in range(n_draft):
        q.append(model.probs(x))
        tokens.append(torch.multinomial(q[-1], 1, generator=g)[:, 0])
        x = model.emb[tokens[-1]]
    tokens, q = torch.stack(tokens, 1), torch.stack(q, 1).view(-1, VOCAB)
    x = model.emb[tokens.flatten()]
    qh, k, v = model.qkv(x)
    p = model.probs(x, cache.attend(qh, k, v, [n_draft + 1] * B))
    accepted, out = torch.empty(B, dtype=torch.int32, device="cuda"), \
        torch.empty(B * (n_draft + 1), dtype=torch.int32, device="cuda")
    noise = torch.empty(B, VOCAB, device="cuda").exponential_(generator=g).clamp_(min=1e-30)
    optr.optr_verify_drafts(cache.p, p, q, tokens[:, 1:].flatten().int(),
                            torch.rand(B * n_draft, device="cuda", generator=g), noise,
                            offsets([n_draft] * B), accepted, out)
    keep = [a + 1 for a in accepted.tolist()]  # the last token and the accepted drafts
    rows = torch.cat([torch.arange(n) + b * (n_draft + 1) for b, n in enumerate(keep)]).cuda()
    cache.write(k[rows], v[rows], keep)
    return [r[:n].tolist() for r, n in zip(out.view(B, -1), keep)]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=24)
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--batch", type=int, default=3)
    ap.add_argument("--prompt", type=int, default=700)
    a = ap.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(0)
    model = Model(1)
    prompts = [a.prompt + 37 * b for b in range(a.batch)]
    limit = max(prompts) + 2 * a.steps * (a.drafts + 1)
    cache = Cache(a.batch, limit, seed=2)
    text = [torch.randint(VOCAB, (n,), device="cuda", generator=g).tolist() for n in prompts]
    done = 0
    while done < max(prompts) - 1:  # all but the last token, 256 a pass
        part = [t[done:min(done + 256, len(t) - 1)] for t in text]
        qh, k, v = model.qkv(model.emb[torch.tensor(sum(part, []), device="cuda")])
        cache.attend(qh, k, v, [len(t) for t in part])  # one layer: only its rows are kept
        cache.write(k, v, [len(t) for t in part])
        done += 256
    counts = []
    for half in range(2):
        made = 0
        for _ in range(a.steps):
            new = step(model, cache, torch.tensor([t[-1] for t in text], device="cuda"), a.drafts, g)
            for t, n in zip(text, new):
                t += n
                made += len(n)
        counts.append(made / (a.steps * a.batch))
        print(f"{made} tokens in {a.steps} steps of {a.batch} sequences, {counts[-1]:.2f} a step")
        if half == 0:  # new rotations, as after a calibration: the cache moves over
            moved = Cache(a.batch, limit, seed=3)
            moved.write(*cache.rows(), cache.len)
            check(cache)
            cache = moved
            print("cache moved to other rotations")
    check(cache)
    return text, cache, counts


if __name__ == "__main__":
    main()
