"""Operators for trees of drafted tokens and for eviction, around the paged INT2 cache, as measurable cases.

* ``tree``: attention of a tree of drafted tokens over the paged cache: a row attends to the sequence's
  cached past (INT2 records, and the BF16 windows where the cache has them), to itself and to its
  ancestors in the tree.
* ``verify``: the tree's drafts verified against the target's probabilities from given random numbers:
  the accepted path, and the token that follows it.
* ``score``: the attention weights that the tokens of a step (or the last ones of a prompt) give to
  every cached position, added to a running sum per (sequence, KV head, position).
* ``select``: the positions that a head keeps: the first and last ones, and of the others those of the
  largest sums.
* ``compact``: the cache's records (their sums, and the windows' ring) moved together over the
  positions that are not kept.

``run()`` computes them in plain torch, in 32 bits and rounded once at the end, or through the library's
entry points where ``own`` is true; ``exact()`` computes them in 64 bits, sequence by sequence.  The cache
is filled here with plain torch (rotated, quantized and packed as include/optr.h lays it out).
"""
from __future__ import annotations

import math
import random

import torch

own = False

D = 128
PAGE = 16
RATIO = 4
DEV = "cuda"

# the paper's cache configuration: G = 128, clips, 64 sink and 256 recent tokens in BF16
PAPER = {"group": 128, "clip_k": 0.96, "clip_v": 0.92, "sink": 64, "recent": 256}
# min-max groups of 32 and no windows: the benchmark's cache
G32 = {"group": 32, "clip_k": 1.0, "clip_v": 1.0, "sink": 0, "recent": 0}


def _tree(B, rows, past, opts, h_kv=8, lens=0):
    return {"op": "tree", "B": B, "new_lo": rows[0], "new_hi": rows[1], "past_lo": past[0],
            "past_hi": past[1], "lens": lens, "h_kv": h_kv, **opts}


def _verify(B, rows, vocab, dtype, sampled, lens=0):
    return {"op": "verify", "B": B, "new_lo": rows[0], "new_hi": rows[1], "vocab": vocab, "dtype": dtype,
            "sampled": sampled, "lens": lens}


def _score(B, new, past, opts, h_kv=8, lens=0):
    return {"op": "score", "B": B, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0], "past_hi": past[1],
            "lens": lens, "h_kv": h_kv, **opts}


def _select(B, lens, keep, first, last, h_kv=8, zeros=0.1, seed=0):
    return {"op": "select", "B": B, "len_lo": lens[0], "len_hi": lens[1], "keep": keep, "first": first,
            "last": last, "h_kv": h_kv, "zeros": zeros, "lens": seed}


def _compact(B, lens, keep, opts, h_kv=8, seed=0):
    return {"op": "compact", "B": B, "len_lo": lens[0], "len_hi": lens[1], "keep": keep, "lens": seed,
            "h_kv": h_kv, **opts}


def listed():
    return [
        # the last token and a tree of seven drafts in one short chat: the smallest call, all latency
        {"name": "tree_1x8_past1k", **_tree(1, (8, 8), (1024, 1024), G32)},
        # trees of many requests, as large as their drafts were sure, in the paper's configuration
        {"name": "tree_ragged_48", **_tree(48, (5, 64), (100, 6001), PAPER, lens=2)},
        # wide trees in the benchmark's serving batch: the largest call
        {"name": "tree_16x61_past8k", **_tree(16, (61, 61), (8192, 8192), G32)},
        # one chat's tree of the draft's likeliest tokens, half-precision probabilities
        {"name": "verify_1x8_32k", **_verify(1, (8, 8), 32000, "bfloat16", False)},
        # the serving batch's trees, drawn from the draft's probabilities, against a large vocabulary
        {"name": "verify_16x24_131k", **_verify(16, (24, 24), 131072, "float32", True)},
        # one new token of one short chat
        {"name": "score_1x1_1k", **_score(1, (1, 1), (1023, 1023), G32)},
        # a decode step of the benchmark's serving batch
        {"name": "score_16x1_8k", **_score(16, (1, 1), (8192, 8192), G32)},
        # the last 64 tokens of two long prompts look over them, in the paper's configuration
        {"name": "score_2x64_32k", **_score(2, (64, 64), (30001, 32704), PAPER, lens=1)},
        # one chat over its budget
        {"name": "select_1x2049", **_select(1, (2049, 2049), 1024, 4, 64)},
        # long ragged contexts cut to a quarter
        {"name": "select_8x32k", **_select(8, (20011, 32768), 8192, 64, 256, seed=4)},
        # a few chats in the paper's configuration, their windows with them
        {"name": "compact_3x1500", **_compact(3, (1100, 1500), 1000, PAPER, seed=3)},
        # the serving batch's caches cut to half
        {"name": "compact_16x8k", **_compact(16, (8192, 8192), 4096, G32)},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    lens = rng.randrange(1 << 20)
    op = rng.choice(["tree", "tree", "verify", "verify", "score", "score", "select", "compact"])
    h_kv = rng.choice([2, 4, 8, 8, 8, 8])
    opts = rng.choice([G32, PAPER, dict(PAPER, sink=0, recent=0), dict(G32, sink=16, recent=100)])
    if op == "verify":
        V = _log(rng, 1000, 152064)
        hi = _log(rng, 1, 64)
        B = _log(rng, 1, max(1, min(64, 50000000 // (hi * V))))
        return _verify(B, (max(1, int(hi * rng.uniform(0.2, 1.0))), hi), V,
                       rng.choice(["float32", "float32", "bfloat16"]), rng.random() < 0.6, lens)
    if op == "select":
        hi = _log(rng, 64, 131072)
        B = _log(rng, 1, max(1, min(64, (1 << 18) // hi)))
        return _select(B, (int(hi * rng.uniform(0.3, 1.0)), hi), max(1, int(hi * rng.uniform(0.05, 0.9))),
                       rng.choice([0, 4, 64]), rng.choice([0, 1, 64, 256]), h_kv,
                       rng.choice([0.0, 0.1, 0.7]), lens)
    if op == "compact":
        hi = _log(rng, 400, 131072)
        B = _log(rng, 1, max(1, min(64, (1 << 17) // hi)))
        return _compact(B, (int(hi * rng.uniform(0.5, 1.0)), hi), max(330, int(hi * rng.uniform(0.1, 0.9))), opts,
                        h_kv, lens)
    if op == "score":
        new = _log(rng, 1, 64)
        B = _log(rng, 1, 64)
        past = _log(rng, 1, min(131072, (1 << 17) // B, (1 << 22) // (B * new)))
        return _score(B, (max(1, int(new * rng.uniform(0.2, 1.0))), new),
                      (int(past * rng.uniform(0.1, 1.0)), past), opts, h_kv, lens)
    new = _log(rng, 1, 200)
    B = _log(rng, 1, 64)
    past = 0 if rng.random() < 0.1 else _log(rng, 1, min(131072, (1 << 17) // B, (1 << 22) // (B * new)))
    return _tree(B, (max(1, int(new * rng.uniform(0.2, 1.0))), new), (int(past * rng.uniform(0.1, 1.0)), past), opts,
                 h_kv, lens)


# ------------------------------------------------------------------ inputs

def _lens(c, lo, hi, stream):
    r = random.Random(c["lens"] * 7 + stream)
    return [r.randint(c[lo], c[hi]) for _ in range(c["B"])]


def _parents(c):
    """The trees' parents, by sequence: row 0 is the root, a row's parent lies in the upper two thirds of
    the rows before it (one or two children a row, some leaves, a depth of ten or so at 64 rows)."""
    r = random.Random(c["lens"] * 7 + 5)
    return [[-1] + [r.randint((i - 1) // 3, i - 1) for i in range(1, n)] for n in _lens(c, "new_lo", "new_hi", 0)]


def _gen(seed, stream):
    return torch.Generator(device=DEV).manual_seed(seed * 1000003 + stream)


def _randn(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


def _ints(x):
    return torch.tensor(x, device=DEV, dtype=torch.int32)


def _cu(lens):
    return torch.tensor([0] + lens).cumsum(0).to(DEV, torch.int32)


def _rotations(h, seed):
    """R_k, R_v [h_kv][128][128] and mu [h_kv][128]: an offset on four channels of each head."""
    g = _gen(seed, 1)
    R = [torch.linalg.qr(_randn(g, h, D, D).double())[0].float() for _ in range(2)]
    off = (torch.rand(h, 4, device=DEV, generator=g) * 4 + 6) * _randn(g, h, 4).sign()
    at = torch.rand(h, D, device=DEV, generator=g).argsort(1)[:, :4]
    return R[0], R[1], torch.zeros(h, D, device=DEV).scatter_(1, at, off)


def _heavy(g, *shape):
    """Student-t, nu = 4."""
    return _randn(g, *shape) / sum(_randn(g, *shape).square() for _ in range(4)).div(4).sqrt()


def _records(z, G, clip):
    """Codes [T][h][32] bytes and {scale, min} [T][h][128 / G][2] fp16 of rotated rows."""
    T, h, _ = z.shape
    x = z.view(T, h, D // G, G)
    mn, mx = x.amin(3, keepdim=True) * clip, x.amax(3, keepdim=True) * clip
    r = (mx - mn).clamp_min(1e-30)
    code = ((x.clamp(mn, mx) - mn) * (3.0 / r)).round().clamp(0, 3).to(torch.uint8)
    code = code.view(T, h, 4, 8, 4)
    byte = (code[..., 0] | code[..., 1] << 2 | code[..., 2] << 4 | code[..., 3] << 6)
    return byte.transpose(2, 3).reshape(T, h, 32), torch.cat((r / 3, mn), 3).half()


def _cache(c, seed, lens, max_pages):
    """A pool filled with `lens` tokens of each sequence on shuffled pages (bytes that no token
    fills are random), its block table, and the window store with its slots (or None)."""
    g = _gen(seed, 2)
    h, G, B = c["h_kv"], c["group"], c["B"]
    rec = 1152 if G == 128 else 1536
    pages = B * max_pages + 3
    pool = torch.randint(0, 256, (pages, h, rec), device=DEV, generator=g, dtype=torch.uint8)
    table = torch.rand(pages, device=DEV, generator=g).argsort()[:B * max_pages].view(B, max_pages).int()
    R_k, R_v, mu = _rotations(h, seed)
    w = c["sink"] + c["recent"]
    slots = torch.rand(B + 2, device=DEV, generator=g).argsort()[:B].int()
    # rows that no position fills hold NaN, as memory that was never written may
    win = torch.full((B + 2, h, 2, w, D), float("nan"), device=DEV, dtype=torch.bfloat16) if w else None
    for b, n in enumerate(lens):
        if n == 0:
            continue
        full = -(-n // PAGE) * PAGE
        k, v = _randn(g, full, h, D), _heavy(g, full, h, D)
        if w:
            s = torch.cat((torch.arange(min(n, c["sink"])), torch.arange(min(n, max(c["sink"], n - c["recent"])), n)))
            row = torch.where(s < c["sink"], s, c["sink"] + (s - c["sink"]) % max(1, c["recent"])).to(DEV)
            s = s.to(DEV)
            at = int(slots[b])
            win[at, :, 0, row] = (k + mu)[s].transpose(0, 1).bfloat16()
            win[at, :, 1, row] = v[s].transpose(0, 1).bfloat16()
        kc, km = _records(torch.einsum("thd,hde->the", k, R_k), G, c["clip_k"])
        vc, vm = _records(torch.einsum("thd,hde->the", v, R_v), G, c["clip_v"])
        parts = [x.view(-1, PAGE, h, x.shape[2:].numel()).transpose(1, 2).flatten(2)
                 for x in (kc, vc, km.flatten(2).view(torch.uint8), vm.flatten(2).view(torch.uint8))]
        pool[table[b, :full // PAGE].long()] = torch.cat(parts, 2)
    return pool, table, win, slots, (R_k, R_v, mu)


def _params(c, rot):
    from paper_2608_02691_gb300 import optr
    R_k, R_v, mu = rot
    return optr.optr_params_create(R_k, R_v, mu, RATIO * c["h_kv"], c["clip_k"], c["clip_v"],
                                   sink=c["sink"], recent=c["recent"], group=c["group"])


def prepare(case, seed):
    return {"tree": _prepare_tree, "verify": _prepare_verify, "score": _prepare_score, "select": _prepare_select,
            "compact": _prepare_compact}[case["op"]](case, seed)


def _prepare_tree(c, seed):
    new, past = _lens(c, "new_lo", "new_hi", 0), _lens(c, "past_lo", "past_hi", 1)
    h, n = c["h_kv"], sum(new)
    pool, table, win, slots, rot = _cache(c, seed, past, -(-(c["past_hi"] + c["new_hi"]) // PAGE))
    g = _gen(seed, 3)
    s = {"c": c, "max_new": max(new), "max_past": max(past), "pool": pool, "table": table, "win": win,
         "slots": slots, "rot": rot, "cu": _cu(new), "pos0": _ints(past), "parent": _ints(sum(_parents(c), [])),
         "q": _randn(g, n, RATIO * h, D).bfloat16(), "k": (_randn(g, n, h, D) + rot[2]).bfloat16(),
         "v": _heavy(g, n, h, D).bfloat16()}
    if own:
        from paper_2608_02691_gb300 import optr
        s["p"] = _params(c, rot)
        s["out"] = torch.empty_like(s["q"])
        s["ws"] = optr.new_chunk_workspace(s["p"], n, c["B"], s["max_new"])
    return s


def _prepare_verify(c, seed):
    """Target and draft distributions that agree on about four tokens in five; a row's children drawn
    independently from its draft distribution."""
    g = _gen(seed, 4)
    trees = _parents(c)
    n, B, V = sum(map(len, trees)), c["B"], c["vocab"]
    dtype = getattr(torch, c["dtype"])
    cu = _cu([len(t) for t in trees])
    z = _randn(g, n, V) * 2.5
    tp = torch.softmax(z, 1).to(dtype)
    dp = torch.softmax(z + 0.5 * _randn(g, n, V), 1).to(dtype)
    parent = _ints(sum(trees, []))
    seq = torch.repeat_interleave(torch.arange(B, device=DEV), cu[1:] - cu[:-1])
    up = (cu[seq] + parent.clamp_min(0)).long()
    tokens = torch.empty(n, device=DEV, dtype=torch.int32)
    for i in range(0, n, 64):
        part = dp[up[i:i + 64]].float()
        e = torch.empty_like(part).exponential_(generator=g).clamp_min(1e-20)
        tokens[i:i + 64] = (part / e).argmax(1).int()
    s = {"c": c, "tp": tp, "dp": dp if c["sampled"] else None, "tokens": tokens, "parent": parent, "cu": cu,
         "depth": max(_depths(t)[1] for t in trees), "u": torch.rand(n, device=DEV, generator=g),
         "noise": torch.empty(B, V, device=DEV).exponential_(generator=g).clamp_min(1e-20)}
    if own:
        i32 = torch.int32
        s["p"] = _params({"h_kv": 8, **G32}, _rotations(8, seed))
        s["accepted"] = torch.empty(B, device=DEV, dtype=i32)
        s["path"], s["next"] = torch.empty(n, device=DEV, dtype=i32), torch.empty(n, device=DEV, dtype=i32)
    return s


def _depths(parents):
    """Rows on the way from the root, itself among them, summed over the tree; the deepest row's."""
    d = []
    for i, p in enumerate(parents):
        d.append(1 if p < 0 else d[p] + 1)
    return sum(d), max(d)


def _prepare_score(c, seed):
    """The step's tokens are in the cache already; the sums hold what earlier steps gave."""
    new, past = _lens(c, "new_lo", "new_hi", 0), _lens(c, "past_lo", "past_hi", 1)
    h, n = c["h_kv"], sum(new)
    lens = [a + b for a, b in zip(past, new)]
    pages = -(-max(lens) // PAGE)
    pool, table, win, slots, rot = _cache(c, seed, lens, pages)
    g = _gen(seed, 3)
    s = {"c": c, "max_new": max(new), "max_len": max(lens), "pool": pool, "table": table, "win": win,
         "slots": slots, "rot": rot, "cu": _cu(new), "pos0": _ints(past),
         "q": (1.5 * _randn(g, n, RATIO * h, D)).bfloat16(),
         "score": torch.rand(c["B"], h, pages * PAGE, device=DEV, generator=g) * (c["new_hi"] * RATIO / c["past_hi"])}
    if own:
        from paper_2608_02691_gb300 import optr
        s["p"] = _params(c, rot)
        s["ws"] = optr.new_score_workspace(s["p"], n, c["B"], s["max_new"], table.shape[1])
    return s


def _prepare_select(c, seed):
    """Sums of heavy tails; some positions were never attended to."""
    lens = _lens(c, "len_lo", "len_hi", 0)
    g = _gen(seed, 5)
    B, h, n = c["B"], c["h_kv"], max(lens)
    score = _heavy(g, B, h, n).abs()
    score = torch.where(torch.rand(B, h, n, device=DEV, generator=g) < c["zeros"], 0.0, score)
    s = {"c": c, "score": score, "lens": _ints(lens), "keep": _ints([c["keep"]] * B),
         "most": min(n, max(c["keep"], c["first"] + c["last"]))}
    if own:
        s["p"] = _params({"h_kv": h, **G32}, _rotations(h, seed))
        s["kept"] = torch.full((B, h, s["most"]), -1, device=DEV, dtype=torch.int32)
        s["n_kept"] = torch.empty(B, device=DEV, dtype=torch.int32)
    return s


def _prepare_compact(c, seed):
    """A list of kept positions for each head: the first and last ones, of the others random ones."""
    lens = _lens(c, "len_lo", "len_hi", 0)
    B, h = c["B"], c["h_kv"]
    pool, table, win, slots, rot = _cache(c, seed, lens, -(-max(lens) // PAGE))
    g = _gen(seed, 6)
    n_kept = [min(n, c["keep"]) for n in lens]
    kept = torch.full((B, h, max(n_kept)), -1, device=DEV, dtype=torch.int32)
    for b, n in enumerate(lens):
        r = torch.rand(h, n, device=DEV, generator=g)
        r[:, :c["sink"]] = 2
        r[:, max(0, n - c["recent"]):n if c["recent"] else 0] = 2
        kept[b, :, :n_kept[b]] = r.topk(n_kept[b], 1).indices.sort(1).values.int()
    s = {"c": c, "pool": pool, "table": table, "win": win, "slots": slots, "rot": rot, "lens": _ints(lens),
         "kept": kept, "n_kept": _ints(n_kept), "score": _heavy(g, B, h, table.shape[1] * PAGE).abs()}
    if own:
        s["p"] = _params(c, rot)
    return s


# ------------------------------------------------------------------ the calls

def run(s):
    op = s["c"]["op"]
    if not own:
        return {"tree": _plain_tree, "verify": _plain_verify, "score": _plain_score, "select": _plain_select,
                "compact": _plain_compact}[op](s)
    from paper_2608_02691_gb300 import optr
    if op == "tree":
        if s["win"] is None:
            optr.optr_tree_attention(s["p"], s["q"], s["k"], s["v"], s["parent"], s["cu"], s["pos0"], s["max_new"],
                                     s["table"], s["pool"], s["out"], s["ws"])
        else:
            optr.optr_tree_attention_win(s["p"], s["q"], s["k"], s["v"], s["parent"], s["cu"], s["pos0"],
                                         s["max_new"], s["table"], s["pool"], s["win"], s["slots"], s["out"],
                                         s["ws"])
        return s["out"]
    if op == "verify":
        optr.optr_verify_tree(s["p"], s["tp"], s["dp"], s["tokens"], s["parent"], s["u"], s["noise"], s["cu"],
                              s["accepted"], s["path"], s["next"])
        return s["accepted"], s["path"], s["next"]
    if op == "score":
        if s["win"] is None:
            optr.optr_kv_score(s["p"], s["q"], s["cu"], s["pos0"], s["max_new"], s["table"], s["pool"], s["score"],
                               s["ws"])
        else:
            optr.optr_kv_score_win(s["p"], s["q"], s["cu"], s["pos0"], s["max_new"], s["table"], s["pool"],
                                   s["win"], s["slots"], s["score"], s["ws"])
        return s["score"]
    if op == "select":
        optr.optr_evict_select(s["p"], s["score"], s["lens"], s["keep"], s["c"]["first"], s["c"]["last"], s["kept"],
                               s["n_kept"])
        return s["kept"], s["n_kept"]
    if s["win"] is None:
        optr.optr_kv_compact(s["p"], s["kept"], s["n_kept"], s["lens"], s["table"], s["pool"], s["score"])
    else:
        optr.optr_kv_compact_win(s["p"], s["kept"], s["n_kept"], s["lens"], s["table"], s["pool"], s["win"],
                                 s["slots"], s["score"])
    return _moved(s)


def _moved(s):
    """The cache after a compaction: the records as they are (moved whole, as words), the sums, the windows."""
    out = [s["pool"].view(torch.int64), s["score"]]
    return out if s["win"] is None else out + [s["win"]]


def _dequant(rec, group):
    """Records [...][1536 or 1152] bytes -> K and V [...][16][128] float32 (rotated)."""
    lead = rec.shape[:-1]
    ng = D // group
    shift = torch.tensor([0, 2, 4, 6], device=DEV, dtype=torch.uint8)
    code = rec[..., :1024].reshape(*lead, 2, PAGE, 8, 4, 1) >> shift & 3
    code = code.transpose(-2, -3).reshape(*lead, 2, PAGE, ng, group)
    meta = rec[..., 1024:].reshape(-1).view(torch.float16).view(*lead, 2, PAGE, ng, 2).float()
    z = (code * meta[..., :1] + meta[..., 1:]).view(*lead, 2, PAGE, D)
    return z.select(-3, 0), z.select(-3, 1)


def _plain_tree(s):
    c = s["c"]
    R_k, R_v, mu = s["rot"]
    B, h, N, sink = c["B"], c["h_kv"], s["max_new"], c["sink"]
    cu, pos0 = s["cu"].long(), s["pos0"].long()
    total = s["q"].shape[0]
    new = cu[1:] - cu[:-1]
    i = torch.arange(N, device=DEV)
    row = (cu[:-1, None] + i).clamp_max(total - 1)
    inside = i < new[:, None]
    q = s["q"][row].float().view(B, N, h, RATIO, D).permute(0, 2, 1, 3, 4).reshape(B, h, N * RATIO, D)
    k, v = (s[x][row].float().transpose(1, 2) for x in "kv")
    v = torch.where(inside[:, None, :, None], v, 0.0)
    scale = 1 / math.sqrt(D)
    # a row sees itself and what its parent sees: paths of twice the length each time
    up = torch.where(inside, s["parent"].long()[row], -1)
    seen = (i[:, None] == i).float() + (up[:, :, None] == i).float()
    length = 1
    while length < N:
        seen, length = ((seen @ seen) > 0).float(), 2 * length
    own_l = q @ (k - mu[:, None]).transpose(2, 3) * scale
    own_l = own_l.masked_fill((seen == 0).repeat_interleave(RATIO, 1)[:, None], -math.inf)
    logits, lens = [own_l], [N]
    P = -(-s["max_past"] // PAGE)
    if P:
        end = (pos0 - c["recent"]).clamp_min(sink)
        K, V = (x.transpose(1, 2).reshape(B, h, P * PAGE, D) for x in
                _dequant(s["pool"][s["table"][:, :P].long()], c["group"]))
        at = torch.arange(P * PAGE, device=DEV)
        cached = ((at >= sink) & (at < end[:, None]))[:, None, None]
        l = (q @ R_k) @ K.transpose(2, 3) * scale
        logits.append(l.masked_fill(~cached, -math.inf))
        V = torch.where(cached.transpose(2, 3), V, 0.0)
        if s["win"] is not None:
            w = s["win"][s["slots"].long()].float()
            filled = (torch.arange(w.shape[3], device=DEV) < pos0[:, None])[:, None, None]
            l = q @ (w[:, :, 0] - mu[:, None]).transpose(2, 3) * scale
            logits.append(l.masked_fill(~filled, -math.inf))
            W = torch.where(filled.transpose(2, 3), w[:, :, 1], 0.0)
    l = torch.cat(logits, 3)
    p = (l - l.amax(3, keepdim=True)).exp()
    p = p / p.sum(3, keepdim=True)
    o = p[..., :N] @ v
    if P:
        o = o + p[..., N:N + P * PAGE] @ V @ R_v.transpose(1, 2)
        if s["win"] is not None:
            o = o + p[..., N + P * PAGE:] @ W
    o = o.view(B, h, N, RATIO, D).transpose(1, 2).reshape(B, N, h * RATIO, D)
    t = torch.arange(total, device=DEV)
    b = torch.searchsorted(cu, t, right=True) - 1
    return o[b, t - cu[b]].bfloat16()


def _plain_verify(s):
    cu, V = s["cu"].long(), s["c"]["vocab"]
    B, n = cu.shape[0] - 1, s["tokens"].shape[0]
    x, dp = s["tokens"].long(), s["dp"]
    t = torch.arange(n, device=DEV)
    seq = torch.searchsorted(cu, t, right=True) - 1
    up = torch.where(s["parent"] >= 0, cu[seq] + s["parent"], -1)
    at = cu[:-1].clone()               # the last accepted row
    path = torch.full((B, s["depth"]), -1, device=DEV)
    path[:, 0] = at
    w, mass = s["tp"][at].float(), torch.ones(B, device=DEV)
    tried = at.clone()                 # children up to this row were rejected
    accepted = torch.zeros(B, device=DEV, dtype=torch.long)
    # one child of each sequence at a time, as many as a sequence has rows at most
    for _ in range(int(s["c"]["new_hi"])):
        child = torch.where((up == at[:, None]) & (t > tried[:, None]), t, n).amin(1)
        open_ = child < n
        child = child.clamp_max(n - 1)
        tok = x[child][:, None]
        q = dp[at].float() if dp is not None else (torch.arange(V, device=DEV) == tok).float()
        qx, wx = q.gather(1, tok)[:, 0], w.gather(1, tok)[:, 0]
        yes = open_ & (s["u"][child] * qx * mass < wx)
        no = open_ & ~yes
        # accepted: on to the child; rejected: what is left of the target
        accepted = accepted + yes
        at = torch.where(yes, child, at)
        path = torch.where(yes[:, None] & (torch.arange(s["depth"], device=DEV) == accepted[:, None]), child[:, None], path)
        if dp is not None:
            left = (w - mass[:, None] * q).clamp_min(0)
            left_mass = left.double().sum(1).float()
        else:
            left, left_mass = w.scatter(1, tok, 0.0), mass - wx
        w = torch.where(yes[:, None], s["tp"][at].float(), torch.where(no[:, None], left, w))
        mass = torch.where(yes, 1.0, torch.where(no, left_mass, mass))
        tried = torch.where(open_, child, tried)
    r = torch.where((w > 0).any(1, keepdim=True), w, s["tp"][at].float())
    token = (r / s["noise"]).argmax(1)
    i = t - cu[seq]
    row = torch.where(i < path.shape[1], path[seq, i.clamp_max(path.shape[1] - 1)], -1)
    after = torch.where(i + 1 < path.shape[1], path[seq, (i + 1).clamp_max(path.shape[1] - 1)], -1)
    out = torch.where(i < accepted[seq], x[after.clamp_min(0)], torch.where(i == accepted[seq], token[seq], -1))
    return accepted.int(), row.int(), out.int()


def _plain_score(s):
    c = s["c"]
    R_k, _, mu = s["rot"]
    B, h, N, sink = c["B"], c["h_kv"], s["max_new"], c["sink"]
    cu, pos0 = s["cu"].long(), s["pos0"].long()
    new = cu[1:] - cu[:-1]
    n = pos0 + new
    i = torch.arange(N, device=DEV)
    row = (cu[:-1, None] + i).clamp_max(s["q"].shape[0] - 1)
    q = s["q"][row].float().view(B, N, h, RATIO, D).permute(0, 2, 1, 3, 4).reshape(B, h, N * RATIO, D)
    scale = 1 / math.sqrt(D)
    P = -(-s["max_len"] // PAGE)
    K = _dequant(s["pool"][s["table"][:, :P].long()], c["group"])[0].transpose(1, 2).reshape(B, h, P * PAGE, D)
    l = (q @ R_k) @ K.transpose(2, 3) * scale
    at = torch.arange(P * PAGE, device=DEV)
    if s["win"] is not None:
        # a window position's logit from its exact key, at the row where the position lies
        ring = torch.where(at < sink, at, sink + (at - sink) % max(1, c["recent"]))
        w = s["win"][s["slots"].long()][:, :, 0].float() - mu[:, None]
        exact_l = (q @ w.transpose(2, 3) * scale)[..., ring]
        l = torch.where(((at < sink) | (at >= (n - c["recent"])[:, None]))[:, None, None], exact_l, l)
    seen = (at <= (pos0[:, None] + i)[:, :, None]) & (i < new[:, None])[:, :, None]
    seen = seen.repeat_interleave(RATIO, 1)[:, None]
    l = l.masked_fill(~seen, -math.inf)
    p = torch.where(seen, (l - l.amax(3, keepdim=True)).exp(), 0.0)
    p = p / p.sum(3, keepdim=True).clamp_min(1e-30)
    s["score"][..., :P * PAGE] += p.sum(2)
    return s["score"]


def _plain_select(s):
    c = s["c"]
    B, h, n = s["score"].shape
    lens, first, last = s["lens"].long()[:, None], c["first"], c["last"]
    n_kept = torch.minimum(lens, torch.maximum(s["keep"].long()[:, None], torch.clamp_max(lens, first + last)))
    at = torch.arange(n, device=DEV)
    always = (at < first) | (at >= lens - last)
    key = s["score"].masked_fill(always[:, None], math.inf).masked_fill((at >= lens)[:, None], -1.0)
    rank = torch.empty(B, h, n, device=DEV, dtype=torch.long)
    rank.scatter_(2, key.sort(dim=2, descending=True, stable=True).indices, at.expand(B, h, n))
    keep = rank < n_kept[:, None]
    place = torch.where(keep, keep.cumsum(2) - 1, s["most"])
    kept = torch.full((B, h, s["most"] + 1), -1, device=DEV, dtype=torch.int32)
    kept.scatter_(2, place, at.int().expand(B, h, n))
    return kept[..., :s["most"]].contiguous(), n_kept[:, 0].int()


def _plain_compact(s):
    c = s["c"]
    B, h, most = s["kept"].shape
    lens, n_kept = s["lens"].long(), s["n_kept"].long()
    i = torch.arange(most, device=DEV)
    b, hh, i = torch.where((i < n_kept[:, None])[:, None].expand(B, h, most))
    src = s["kept"][b, hh, i].long()
    table = s["table"].long()
    sizes = (32, 32, 4, 4) if c["group"] == 128 else (32, 32, 16, 16)
    lo = 0
    for size in sizes:  # a record's codes and pairs, slot by slot
        part = s["pool"][..., lo:lo + PAGE * size].unflatten(2, (PAGE, size))
        part[table[b, i // PAGE], hh, i % PAGE] = part[table[b, src // PAGE], hh, src % PAGE]
        lo += PAGE * size
    moved = s["score"][b, hh, src]
    at = torch.arange(s["score"].shape[2], device=DEV)
    s["score"].masked_fill_(((at >= n_kept[:, None]) & (at < lens[:, None]))[:, None], 0.0)
    s["score"][b, hh, i] = moved
    if s["win"] is not None and c["recent"]:
        sink, recent = c["sink"], c["recent"]
        j = torch.arange(recent, device=DEV)
        pos = lens[:, None] - 1 - j          # the recent window's positions, old and new
        b, j = torch.where((pos >= sink) & (lens > n_kept)[:, None])
        pos, slot = pos[b, j], s["slots"].long()[b]
        to = sink + (pos - (lens - n_kept)[b] - sink) % recent
        s["win"][slot, :, :, to] = s["win"][slot, :, :, sink + (pos - sink) % recent]
    return _moved(s)


def work(c):
    if c["op"] == "verify":
        # the target's row that the token is drawn from and the noise of it; with probabilities, where a
        # child is rejected (about one in five), the draft's row too; a probability of each draft
        n = sum(_lens(c, "new_lo", "new_hi", 0))
        size = 4 if c["dtype"] == "float32" else 2
        rows = c["vocab"] * c["B"] * (size + 4 + (0.5 * size if c["sampled"] else 0))
        return {"bytes": int(rows + n * (2 * size + 16) + 4 * c["B"]), "flops": int(c["vocab"] * c["B"] * 3)}
    h = c["h_kv"]
    if c["op"] == "select":
        lens = _lens(c, "len_lo", "len_hi", 0)
        kept = sum(min(n, max(c["keep"], c["first"] + c["last"])) for n in lens)
        return {"bytes": 4 * h * (sum(lens) + kept), "flops": h * sum(lens)}
    rec = 72 if c["group"] == 128 else 96
    if c["op"] == "compact":
        lens = _lens(c, "len_lo", "len_hi", 0)
        kept = sum(min(n, c["keep"]) for n in lens)
        ring = sum(c["recent"] for n in lens if n > c["keep"])
        return {"bytes": h * ((2 * rec + 8) * (kept - c["B"] * c["sink"]) + 4 * sum(lens) + 4 * kept + 1024 * ring),
                "flops": 0}
    new, past = _lens(c, "new_lo", "new_hi", 0), _lens(c, "past_lo", "past_hi", 1)
    size, flops = 0, 0
    if c["op"] == "score":
        for n, s in zip(new, past):
            t = s + n
            win = min(t, c["sink"] + c["recent"])
            size += h * ((t - win) * rec // 2 + win * 2 * D + 8 * t) + n * h * RATIO * 2 * D
            flops += h * RATIO * 2 * D * (n * s + n * (n + 1) // 2 + D * n * (t > win))
        return {"bytes": size, "flops": flops}
    for n, s, parents in zip(new, past, _parents(c)):
        coded = max(0, s - c["recent"] - c["sink"]) if c["recent"] else max(0, s - c["sink"])
        size += h * (coded * rec + (s - coded) * 4 * D + n * 4 * D) + n * h * RATIO * 4 * D + 4 * n
        flops += h * RATIO * (4 * D * (n * s + _depths(parents)[0]) + 2 * 2 * D * D * n * (coded > 0))
    return {"bytes": size, "flops": flops}


# ------------------------------------------------------------------ 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"tree": _exact_tree, "verify": _exact_verify, "score": _exact_score, "select": _exact_select,
            "compact": _exact_compact}[case["op"]](s)


def _row64(s, b, h, lo, hi, kind):
    """Positions lo .. hi-1 of a head's cached keys (kind 0) or values (1), rotated basis."""
    c = s["c"]
    pos = torch.arange(lo, hi, device=DEV)
    rec = s["pool"][s["table"][b].long()[pos // PAGE], h]
    slot = (pos % PAGE)[:, None]
    ch = torch.arange(D, device=DEV)
    byte = 512 * kind + 32 * slot + 4 * (ch % 32 // 4) + ch // 32
    code = rec.gather(1, byte).long() // 4 ** (ch % 4) % 4
    ng = D // c["group"]
    base = 1024 + 64 * ng * kind + 4 * ng * slot + 4 * (ch // c["group"])

    def half(off):
        lohi = torch.stack((rec.gather(1, base + off), rec.gather(1, base + off + 1)), 2)
        return lohi.view(torch.float16)[..., 0].double()

    return code * half(0) + half(2)


def _model64(s, b, h, n, values=True):
    """The first n positions' keys (centered) and values of a head in the model's basis, in order: window
    positions of a sequence of n tokens from their exact rows, the others from their records."""
    c = s["c"]
    R_k, R_v, mu = (x.double() for x in s["rot"])
    out = []
    for kind, R in ((0, R_k), (1, R_v))[:1 + values]:
        x = _row64(s, b, h, 0, n, kind) @ R[h].T
        if s["win"] is not None:
            pos = torch.arange(n, device=DEV)
            pos = pos[(pos < c["sink"]) | (pos >= n - c["recent"])]
            row = torch.where(pos < c["sink"], pos, c["sink"] + (pos - c["sink"]) % max(1, c["recent"]))
            w = s["win"][int(s["slots"][b]), h, kind][row].double()
            x[pos] = w - mu[h] if kind == 0 else w
        out.append(x)
    return out


def _exact_tree(s):
    c = s["c"]
    mu = s["rot"][2].double()
    cu, past, parent = s["cu"].tolist(), s["pos0"].tolist(), s["parent"].tolist()
    out = torch.empty_like(s["q"], dtype=torch.float64)
    for b in range(c["B"]):
        r0, r1, n = cu[b], cu[b + 1], past[b]
        seen = []
        for i, p in enumerate(parent[r0:r1]):
            seen.append((set() if p < 0 else seen[p]) | {i})
        mask = torch.tensor([[j in x for j in range(r1 - r0)] for x in seen], device=DEV)
        for h in range(c["h_kv"]):
            K, V = _model64(s, b, h, n)
            K = torch.cat((K, s["k"][r0:r1, h].double() - mu[h]))
            V = torch.cat((V, s["v"][r0:r1, h].double()))
            for j in range(RATIO):
                l = s["q"][r0:r1, RATIO * h + j].double() @ K.T / D ** 0.5
                l[:, n:].masked_fill_(~mask, -math.inf)
                out[r0:r1, RATIO * h + j] = torch.softmax(l, 1) @ V
    return out


def _exact_verify(s):
    cu, x, u, parent = s["cu"].tolist(), s["tokens"].tolist(), s["u"].double().tolist(), s["parent"].tolist()
    first, path, out = [], [], []
    for b in range(len(cu) - 1):
        lo, hi = cu[b], cu[b + 1]
        way = [lo]
        while True:
            r = way[-1]
            w, total = s["tp"][r].double(), 1.0
            step = None
            for c in range(lo, hi):
                if parent[c] != r - lo:
                    continue
                if s["dp"] is not None:
                    q = s["dp"][r].double()
                else:
                    q = torch.zeros_like(w)
                    q[x[c]] = 1
                if u[c] * float(q[x[c]]) * total < float(w[x[c]]):
                    step = c
                    break
                if s["dp"] is not None:
                    w = (w - total * q).clamp_min(0)
                    total = float(w.sum())
                else:
                    total -= float(w[x[c]])
                    w = w.clone()
                    w[x[c]] = 0
            if step is None:
                break
            way.append(step)
        if not bool((w > 0).any()):
            w = s["tp"][r].double()
        token = int((w / s["noise"][b].double()).argmax())
        n, a = hi - lo, len(way) - 1
        first.append(a)
        path += way + [-1] * (n - 1 - a)
        out += [x[c] for c in way[1:]] + [token] + [-1] * (n - 1 - a)
    return _ints(first), _ints(path), _ints(out)


def _exact_score(s):
    c = s["c"]
    cu, past = s["cu"].tolist(), s["pos0"].tolist()
    out = s["score"].double()
    for b in range(c["B"]):
        r0, r1 = cu[b], cu[b + 1]
        n = past[b] + r1 - r0
        i = torch.arange(r1 - r0, device=DEV)[:, None]
        for h in range(c["h_kv"]):
            K, = _model64(s, b, h, n, values=False)
            for j in range(RATIO):
                l = s["q"][r0:r1, RATIO * h + j].double() @ K.T / D ** 0.5
                l = l.masked_fill(torch.arange(n, device=DEV) > past[b] + i, -math.inf)
                out[b, h, :n] += torch.softmax(l, 1).sum(0)
    return out


def _exact_select(s):
    c = s["c"]
    score = s["score"].double().cpu()
    lens, keep = s["lens"].tolist(), s["keep"].tolist()
    kept = torch.full((c["B"], c["h_kv"], s["most"]), -1, dtype=torch.int32)
    counts = []
    for b, n in enumerate(lens):
        m = min(n, max(keep[b], min(n, c["first"] + c["last"])))
        counts.append(m)
        for h in range(c["h_kv"]):
            ends = set(range(min(n, c["first"]))) | set(range(max(0, n - c["last"]), n))
            x = score[b, h, :n].tolist()
            others = sorted((p for p in range(n) if p not in ends), key=lambda p: (-x[p], p))
            kept[b, h, :m] = torch.tensor(sorted(list(ends) + others[:m - len(ends)]), dtype=torch.int32)
    return kept.to(DEV), _ints(counts)


def _exact_compact(s):
    c = s["c"]
    lens, n_kept, table, slots = (s[x].tolist() for x in ("lens", "n_kept", "table", "slots"))
    pool, score = s["pool"].clone(), s["score"].double()
    win = None if s["win"] is None else s["win"].double()
    rec = 72 if c["group"] == 128 else 96
    meta = (rec - 64) // 2
    # each byte of a slot's record, by its place in the page's
    place = torch.cat([base + size * torch.arange(PAGE)[:, None] + torch.arange(size) for base, size in
                       ((0, 32), (512, 32), (1024, meta), (1024 + PAGE * meta, meta))], 1).to(DEV)
    for b, (n, m) in enumerate(zip(lens, n_kept)):
        pages = torch.tensor(table[b], device=DEV)
        for h in range(c["h_kv"]):
            kept = s["kept"][b, h, :m].long()
            new = torch.arange(m, device=DEV)
            pool[pages[new // PAGE][:, None], h, place[new % PAGE]] = \
                s["pool"][pages[kept // PAGE][:, None], h, place[kept % PAGE]]
            score[b, h, :n] = 0
            score[b, h, :m] = s["score"][b, h, kept].double()
        if win is not None and m < n:
            for pos in range(max(c["sink"], n - c["recent"]), n):
                old, new = (c["sink"] + (x - c["sink"]) % c["recent"] for x in (pos, pos - (n - m)))
                win[slots[b], :, :, new] = s["win"][slots[b], :, :, old].double()
    out = [pool.view(torch.int64), score]
    return out if win is None else out + [win]
