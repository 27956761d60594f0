"""Three operators around the paged INT2 cache, as measurable cases.

* ``chunk``: attention of a chunk of new tokens over the paged cache.  The
  queries of every sequence's new tokens attend to the sequence's cached past
  (INT2 records, and the BF16 windows where the cache has them) and, causally,
  to the chunk's own keys and values as given.
* ``read``: cached rows read back, dequantized and rotated into the model's
  basis.
* ``verify``: drafted tokens verified against the target's probabilities from
  given random numbers, with the token that replaces the first rejected one
  (or follows the last accepted one).

``run()`` computes them in plain torch, in 32 bits and rounded once at the
end, or through the library's entry points where ``own`` is true; ``exact()``
computes them in 64 bits, sequence by sequence.  The cache is filled here with
plain torch (rotated, quantized and packed as include/optr.h lays it out).
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


def _chunk(B, new, past, opts, h_kv=8, fold=False, lens=0):
    return {"op": "chunk", "B": B, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0],
            "past_hi": past[1], "lens": lens, "h_kv": h_kv, "fold": fold, **opts}


def _read(B, lo, hi, first, opts, h_kv=8, fold=False, lens=0):
    return {"op": "read", "B": B, "len_lo": lo, "len_hi": hi, "first": first, "lens": lens,
            "h_kv": h_kv, "fold": fold, **opts}


def _verify(B, drafts, vocab, dtype, sampled, lens=0):
    return {"op": "verify", "B": B, "draft_lo": drafts[0], "draft_hi": drafts[1], "vocab": vocab,
            "dtype": dtype, "sampled": sampled, "lens": lens}


def listed():
    return [
        # one new token of one short chat: the smallest call, all latency
        {"name": "chunk_1x1_past1k", **_chunk(1, (1, 1), (1024, 1024), G32)},
        # four drafts and the token before them, in the benchmark's serving batch
        {"name": "chunk_16x5_past8k", **_chunk(16, (5, 5), (8192, 8192), G32)},
        # the same over one long context, which only a split along it can fill the GPU with
        {"name": "chunk_1x8_past128k", **_chunk(1, (8, 8), (131072, 131072), G32)},
        # ragged drafts of many requests in the paper's configuration
        {"name": "chunk_ragged_64", **_chunk(64, (1, 9), (100, 6001), PAPER, lens=2)},
        # one chunk of a chunked prefill in the paper's configuration
        {"name": "chunk_2000_past4k", **_chunk(1, (2000, 2000), (4096, 4096), PAPER)},
        # a whole prompt: nothing is cached yet
        {"name": "chunk_8192_first", **_chunk(1, (8192, 8192), (0, 0), G32)},
        # a later chunk of a long prompt: the largest call
        {"name": "chunk_2048_past32k", **_chunk(1, (2048, 2048), (32768, 32768), G32)},
        # a short cached prefix of one chat handed on to another model instance
        {"name": "read_1x777", **_read(1, 777, 777, 5, PAPER)},
        # a serving batch's caches moved to newly calibrated rotations
        {"name": "read_16x8k", **_read(16, 8192, 8192, 0, G32)},
        # one chat's drafts, half-precision probabilities, drafted without probabilities
        {"name": "verify_1x4_32k", **_verify(1, (4, 4), 32000, "bfloat16", False)},
        # the serving batch's drafts against a large vocabulary
        {"name": "verify_16x4_131k", **_verify(16, (4, 4), 131072, "float32", True)},
        # a full ragged batch and a vocabulary of odd size
        {"name": "verify_ragged_128", **_verify(128, (0, 8), 100003, "float32", True, lens=3)},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    lens = rng.randrange(1 << 20)
    op = rng.choice(["chunk", "chunk", "chunk", "chunk", "read", "verify", "verify"])
    if op == "verify":
        lo, hi = sorted((rng.randint(0, 8), rng.randint(1, 8)))
        return _verify(_log(rng, 1, 128), (lo, hi), _log(rng, 1000, 152064),
                       rng.choice(["float32", "float32", "bfloat16"]), rng.random() < 0.7, lens)
    opts = rng.choice([G32, PAPER, dict(PAPER, sink=0, recent=0), dict(G32, sink=16, recent=100)])
    h_kv = rng.choice([2, 4, 8, 8, 8, 8])
    fold = rng.random() < 0.25
    if op == "read":
        n = _log(rng, 1, 131072)
        B = min(n, _log(rng, 1, 64))
        return _read(B, max(1, int(n // B * rng.uniform(0.3, 1.0))), n // B,
                     rng.choice([0, rng.randint(0, 4000)]), opts, h_kv, fold, lens)
    # the drafts of a batch, or one chunk of a prefill (of few sequences)
    if rng.random() < 0.5:
        B, new = _log(rng, 1, 128), _log(rng, 1, 16)
    else:
        B, new = rng.choice([1, 1, 1, 2, 3]), _log(rng, 17, 4096)
    most = min(131072, (1 << 18) // B, (1 << 26) // (B * new))
    past = 0 if rng.random() < 0.15 else _log(rng, 1, most)
    lo = past if rng.random() < 0.4 else int(past * rng.uniform(0.05, 1.0))
    return _chunk(B, (max(1, int(new * rng.uniform(0.2, 1.0))), new), (lo, past), opts, h_kv, fold, lens)


# ------------------------------------------------------------------ inputs

def _lens(c, lo, hi, stream):
    r = random.Random(c["lens"] * 7 + stream)
    return [r.randint(c[lo], c[hi]) for _ in range(c["B"])]


def _gen(seed, stream):
    return torch.Generator(device=DEV).manual_seed(seed * 1000003 + stream)


def _randn(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


def _cu(lens):
    return torch.tensor([0] + lens).cumsum(0).to(DEV, torch.int32)


def _rotations(c, seed):
    """R_k, R_v [h_kv][128][128] (R_v None where it is folded) and mu [h_kv][128]: an offset on
    four channels of each head."""
    g = _gen(seed, 1)
    h = c["h_kv"]
    R = [torch.linalg.qr(_randn(g, h, D, D).double())[0].float() for _ in range(2)]
    off = (torch.rand(h, 4, device=DEV, generator=g) * 4 + 6) * _randn(g, h, 4).sign()
    at = torch.rand(h, D, device=DEV, generator=g).argsort(1)[:, :4]
    mu = torch.zeros(h, D, device=DEV).scatter_(1, at, off)
    return R[0], None if c["fold"] else R[1], mu


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
    R_k, R_v, mu = _rotations(c, seed)
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
            s = torch.cat((torch.arange(min(n, c["sink"])), torch.arange(max(c["sink"], n - c["recent"]), n)))
            row = torch.where(s < c["sink"], s, c["sink"] + (s - c["sink"]) % max(1, c["recent"])).to(DEV)
            s = s.to(DEV)
            at = int(slots[b])
            win[at, :, 0, row] = (k + mu)[s].transpose(0, 1).bfloat16()
            win[at, :, 1, row] = v[s].transpose(0, 1).bfloat16()
        kc, km = _records(torch.einsum("thd,hde->the", k, R_k), G, c["clip_k"])
        vc, vm = _records(v if R_v is None else torch.einsum("thd,hde->the", v, R_v), G, c["clip_v"])
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
    return {"chunk": _prepare_chunk, "read": _prepare_read, "verify": _prepare_verify}[case["op"]](case, seed)


def _prepare_chunk(c, seed):
    new, past = _lens(c, "new_lo", "new_hi", 0), _lens(c, "past_lo", "past_hi", 1)
    h, n = c["h_kv"], sum(new)
    max_pages = -(-(c["past_hi"] + c["new_hi"]) // PAGE)
    pool, table, win, slots, rot = _cache(c, seed, past, max_pages)
    g = _gen(seed, 3)
    s = {"c": c, "max_new": max(new), "max_past": max(past), "pool": pool, "table": table, "win": win,
         "slots": slots, "rot": rot, "cu": _cu(new), "pos0": torch.tensor(past, device=DEV, dtype=torch.int32),
         "q": _randn(g, n, RATIO * h, D).bfloat16(), "k": (_randn(g, n, h, D) + rot[2]).bfloat16(),
         "v": _heavy(g, n, h, D).bfloat16()}
    if own:
        from paper_2608_02691_gb300 import optr
        s["p"] = _params(c, rot)
        s["out"] = torch.empty_like(s["q"])
        s["ws"] = optr.new_chunk_workspace(s["p"], n, c["B"], s["max_new"])
    return s


def _prepare_read(c, seed):
    lens = _lens(c, "len_lo", "len_hi", 0)
    last = [c["first"] + n for n in lens]
    pool, table, win, slots, rot = _cache(c, seed, last, -(-max(last) // PAGE))
    n = sum(lens)
    s = {"c": c, "n": n, "pool": pool, "table": table, "rot": rot, "cu": _cu(lens),
         "pos0": torch.full((c["B"],), c["first"], device=DEV, dtype=torch.int32)}
    if own:
        s["p"] = _params(c, rot)
        s["k"], s["v"] = (torch.empty(n, c["h_kv"], D, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    return s


def _prepare_verify(c, seed):
    """Target and draft distributions that agree on about four tokens in five; drafts drawn from
    the draft distribution."""
    g = _gen(seed, 4)
    lens = _lens(c, "draft_lo", "draft_hi", 0)
    n, B, V = sum(lens), c["B"], c["vocab"]
    dtype = getattr(torch, c["dtype"])
    cu = _cu(lens)
    z = _randn(g, n + B, V) * 2.5
    tp = torch.softmax(z, 1).to(dtype)
    rows = torch.tensor([cu_b + b + i for b, cu_b in enumerate(cu.tolist()[:-1]) for i in range(lens[b])],
                        device=DEV, dtype=torch.long)
    dp = torch.softmax(z[rows] + 0.5 * _randn(g, n, V), 1).to(dtype)
    drafts = (dp.float() / torch.empty_like(dp, dtype=torch.float32).exponential_(generator=g).clamp_min(1e-20)).argmax(1).int()
    s = {"c": c, "tp": tp, "dp": dp if c["sampled"] else None, "drafts": drafts, "cu": cu,
         "u": torch.rand(n, device=DEV, generator=g),
         "noise": torch.empty(B, V, device=DEV).exponential_(generator=g).clamp_min(1e-20)}
    if own:
        from paper_2608_02691_gb300 import optr
        i32 = torch.int32
        rot = _rotations({"h_kv": 8, "fold": False}, seed)
        s["p"] = _params({"h_kv": 8, **G32}, rot)
        s["accepted"] = torch.empty(B, device=DEV, dtype=i32)
        s["tokens"] = torch.empty(n + B, device=DEV, dtype=i32)
    return s


# ------------------------------------------------------------------ the calls

def run(s):
    op = s["c"]["op"]
    if not own:
        return {"chunk": _plain_chunk, "read": _plain_read, "verify": _plain_verify}[op](s)
    from paper_2608_02691_gb300 import optr
    if op == "chunk":
        if s["win"] is None:
            optr.optr_chunk_attention(s["p"], s["q"], s["k"], s["v"], s["cu"], s["pos0"], s["max_new"],
                                      s["table"], s["pool"], s["out"], s["ws"])
        else:
            optr.optr_chunk_attention_win(s["p"], s["q"], s["k"], s["v"], s["cu"], s["pos0"], s["max_new"],
                                          s["table"], s["pool"], s["win"], s["slots"], s["out"], s["ws"])
        return s["out"]
    if op == "read":
        optr.optr_kv_read(s["p"], s["cu"], s["pos0"], s["table"], s["pool"], s["k"], s["v"])
        return s["k"], s["v"]
    optr.optr_verify_drafts(s["p"], s["tp"], s["dp"], s["drafts"], s["u"], s["noise"], s["cu"],
                            s["accepted"], s["tokens"])
    return s["accepted"], s["tokens"]


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


def _plain_chunk(s):
    c = s["c"]
    R_k, R_v, mu = s["rot"]
    B, h, N, sink = c["B"], c["h_kv"], s["max_new"], c["sink"]
    cu, pos0 = s["cu"].long(), s["pos0"].long()
    total = s["q"].shape[0]
    new = cu[1:] - cu[:-1]
    i = torch.arange(N, device=DEV)
    row = (cu[:-1, None] + i).clamp_max(total - 1)
    q = s["q"][row].float().view(B, N, h, RATIO, D).permute(0, 2, 1, 3, 4).reshape(B, h, N * RATIO, D)
    k, v = (s[x][row].float().transpose(1, 2) for x in "kv")
    v = torch.where((i < new[:, None])[:, None, :, None], v, 0.0)
    scale = 1 / math.sqrt(D)
    # the chunk itself, causal
    own_l = q @ (k - mu[:, None]).transpose(2, 3) * scale
    seen = (i <= i[:, None]) & (i < new[:, None, None])
    own_l = own_l.masked_fill(~seen.repeat_interleave(RATIO, 1)[:, None], -math.inf)
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
        r = p[..., N:N + P * PAGE] @ V
        o = o + (r if R_v is None else r @ R_v.transpose(1, 2))
        if s["win"] is not None:
            o = o + p[..., N + P * PAGE:] @ W
    o = o.view(B, h, N, RATIO, D).transpose(1, 2).reshape(B, N, h * RATIO, D)
    t = torch.arange(total, device=DEV)
    b = torch.searchsorted(cu, t, right=True) - 1
    return o[b, t - cu[b]].bfloat16()


def _plain_read(s):
    c = s["c"]
    R_k, R_v, mu = s["rot"]
    K, V = (x.transpose(1, 2) for x in _dequant(s["pool"], c["group"]))
    cu = s["cu"].long()
    t = torch.arange(s["n"], device=DEV)
    b = torch.searchsorted(cu, t, right=True) - 1
    pos = s["pos0"].long()[b] + t - cu[b]
    page = s["table"].long()[b, pos // PAGE]
    k, v = K[page, pos % PAGE], V[page, pos % PAGE]
    k = torch.einsum("thd,hed->the", k, R_k) + mu
    if R_v is not None:
        v = torch.einsum("thd,hed->the", v, R_v)
    return k.bfloat16(), v.bfloat16()


def _plain_verify(s):
    cu, V = s["cu"].long(), s["c"]["vocab"]
    B, n = cu.shape[0] - 1, s["drafts"].shape[0]
    x = s["drafts"].long()
    t = torch.arange(n, device=DEV)
    b = torch.searchsorted(cu, t, right=True) - 1
    px = s["tp"][t + b, x].float()
    qx = s["dp"][t, x].float() if s["dp"] is not None else torch.ones_like(px)
    rejected = ~(s["u"] * qx < px)
    # the first rejected draft of each sequence, or its number of drafts
    first = (cu[1:] - cu[:-1]).scatter_reduce(0, b, torch.where(rejected, t - cu[b], n + 1), "amin")
    seq = torch.arange(B, device=DEV)
    at = cu[:-1] + first
    whole = at == cu[1:]
    p = s["tp"][at + seq].float()
    r = p
    if n:
        d = at.clamp_max(n - 1)
        q = s["dp"][d].float() if s["dp"] is not None else p * (torch.arange(V, device=DEV) == x[d][:, None])
        r = torch.where(whole[:, None], p, (p - q).clamp_min(0))
        r = torch.where((r > 0).any(1, keepdim=True), r, p)
    token = (r / s["noise"]).argmax(1).int()
    # accepted drafts, the sampled token, -1
    rows = torch.arange(n + B, device=DEV)
    start = cu + torch.arange(B + 1, device=DEV)
    sb = torch.searchsorted(start, rows, right=True) - 1
    i = rows - start[sb]
    out = torch.where(i == first[sb], token[sb], -1)
    if n:
        out = torch.where(i < first[sb], s["drafts"][(cu[sb] + i).clamp_max(n - 1)], out)
    return first.int(), out.int()


def work(c):
    if c["op"] == "verify":
        # the target's row that the token is drawn from and the noise of it; the draft's row where
        # a draft is rejected (about one in five); a probability of each draft
        lens = _lens(c, "draft_lo", "draft_hi", 0)
        size = 4 if c["dtype"] == "float32" else 2
        rejected = sum(1 - 0.8 ** n for n in lens) if c["sampled"] else 0
        rows = c["vocab"] * (len(lens) * (size + 4) + rejected * size)
        return {"bytes": int(rows + sum(lens) * (2 * size + 12) + 12 * c["B"]),
                "flops": int(c["vocab"] * (2 * len(lens) + rejected))}
    rec = 72 if c["group"] == 128 else 96
    h = c["h_kv"]
    if c["op"] == "read":
        n = sum(_lens(c, "len_lo", "len_hi", 0))
        return {"bytes": n * h * (rec + 4 * D), "flops": n * h * (1 if c["fold"] else 2) * 2 * D * D}
    new, past = _lens(c, "new_lo", "new_hi", 0), _lens(c, "past_lo", "past_hi", 1)
    size, flops = 0, 0
    for n, s in zip(new, past):
        coded = max(0, s - c["recent"] - c["sink"]) if c["recent"] else max(0, s - c["sink"])
        size += h * (coded * rec + (s - coded) * 4 * D + n * 4 * D) + n * h * RATIO * 4 * D
        flops += h * RATIO * (4 * D * (n * s + n * (n + 1) // 2) + (2 - c["fold"]) * 2 * D * D * n * (coded > 0))
    return {"bytes": size, "flops": flops}


# ------------------------------------------------------------------ 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"chunk": _exact_chunk, "read": _exact_read, "verify": _exact_verify}[case["op"]](s)


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


def _exact_chunk(s):
    c = s["c"]
    R_k, R_v, mu = (None if x is None else x.double() for x in s["rot"])
    cu, past = s["cu"].tolist(), s["pos0"].tolist()
    out = torch.empty_like(s["q"], dtype=torch.float64)
    for b in range(c["B"]):
        r0, r1, n = cu[b], cu[b + 1], past[b]
        end = max(c["sink"], n - c["recent"])
        for h in range(c["h_kv"]):
            k = s["k"][r0:r1, h].double() - mu[h]
            v = s["v"][r0:r1, h].double()
            m = n
            if s["win"] is not None and n:
                w = s["win"][int(s["slots"][b]), h, :, :min(n, c["sink"] + c["recent"])].double()
                k, v = torch.cat((w[0] - mu[h], k)), torch.cat((w[1], v))
                m = w.shape[1]
                n_int = max(0, end - c["sink"])
            else:
                n_int = n
            if n_int:
                ck = _row64(s, b, h, c["sink"], c["sink"] + n_int, 0)
                cv = _row64(s, b, h, c["sink"], c["sink"] + n_int, 1)
                k = torch.cat((ck @ R_k[h].T, k))
                v = torch.cat((cv if R_v is None else cv @ R_v[h].T, v))
                m = k.shape[0] - (r1 - r0)
            i = torch.arange(r1 - r0, device=DEV)
            for j in range(RATIO):
                q = s["q"][r0:r1, RATIO * h + j].double()
                l = q @ k.T / D ** 0.5
                l[:, m:].masked_fill_(i > i[:, None], -math.inf)
                out[r0:r1, RATIO * h + j] = torch.softmax(l, 1) @ v
    return out


def _exact_read(s):
    R_k, R_v, mu = (None if x is None else x.double() for x in s["rot"])
    cu, first = s["cu"].tolist(), s["pos0"].tolist()
    h_kv = s["c"]["h_kv"]
    k, v = (torch.empty(s["n"], h_kv, D, device=DEV, dtype=torch.float64) for _ in range(2))
    for b in range(s["c"]["B"]):
        lo, hi = first[b], first[b] + cu[b + 1] - cu[b]
        for h in range(h_kv):
            k[cu[b]:cu[b + 1], h] = _row64(s, b, h, lo, hi, 0) @ R_k[h].T + mu[h]
            z = _row64(s, b, h, lo, hi, 1)
            v[cu[b]:cu[b + 1], h] = z if R_v is None else z @ R_v[h].T
    return k, v


def _exact_verify(s):
    cu, drafts, u = s["cu"].tolist(), s["drafts"].tolist(), s["u"].double().tolist()
    first, out = [], []
    for b in range(len(cu) - 1):
        n, a = cu[b + 1] - cu[b], 0
        while a < n:
            x = drafts[cu[b] + a]
            q = float(s["dp"][cu[b] + a, x]) if s["dp"] is not None else 1.0
            if not u[cu[b] + a] * q < float(s["tp"][cu[b] + b + a, x]):
                break
            a += 1
        p = s["tp"][cu[b] + b + a].double()
        r = p
        if a < n:
            if s["dp"] is not None:
                r = (p - s["dp"][cu[b] + a].double()).clamp_min(0)
            else:
                r = p.clone()
                r[drafts[cu[b] + a]] = 0
            if not bool((r > 0).any()):
                r = p
        token = int((r / s["noise"][b].double()).argmax())
        first.append(a)
        out += drafts[cu[b]:cu[b] + a] + [token] + [-1] * (n - a)
    i32 = torch.int32
    return torch.tensor(first, device=DEV, dtype=i32), torch.tensor(out, device=DEV, dtype=i32)
