"""Attention over the states of an encoder and over a paged 8-bit key/value cache, with what keeps that cache.

Four operators, each as a user's program calls it (`own`) and in its plain form:

  encoder  attention of B x nq queries to the 16-bit states of an encoder: another length, one per request;
  plan     block tables and slot maps of a paged cache, built from the requests' lengths;
  write    rows of keys and values into the cache (8-bit codes, one scale for each page and head), and back out as the
           values that the codes stand for;
  cached   attention over that cache.

Lengths of a case are spread evenly between two numbers, whatever the seed; the seed decides which request has which.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------------ cases
def _encoder(name, batch, heads, kv_heads, nq, nk, d, dtype, lo, fused):
    """lo: shortest length (nk: all are full); fused: keys and values are views of one projection's output."""
    return dict(name=name, kind="encoder", batch=batch, heads=heads, kv_heads=kv_heads, nq=nq, nk=nk, d=d, dtype=dtype,
                lo=lo, fused=fused)


def _plan(name, batch, page, len_lo, len_hi, new_lo, new_hi):
    return dict(name=name, kind="plan", batch=batch, page=page, len_lo=len_lo, len_hi=len_hi, new_lo=new_lo, new_hi=new_hi)


def _write(name, batch, kv_heads, d, page, dtype, len_lo, len_hi, new_lo, new_hi):
    return dict(name=name, kind="write", batch=batch, kv_heads=kv_heads, d=d, page=page, dtype=dtype, len_lo=len_lo,
                len_hi=len_hi, new_lo=new_lo, new_hi=new_hi)


def _cached(name, batch, heads, kv_heads, nq_lo, nq_hi, len_lo, len_hi, d, page, dtype, causal):
    return dict(name=name, kind="cached", batch=batch, heads=heads, kv_heads=kv_heads, nq_lo=nq_lo, nq_hi=nq_hi,
                len_lo=len_lo, len_hi=len_hi, d=d, page=page, dtype=dtype, causal=causal)


def listed():
    return [
        # The 64x64 level of the UNet at batch 2 (classifier-free guidance) over 77 text tokens, full-precision scores.
        _encoder("encoder_2x8x4096x40_text77_f16", 2, 8, 8, 4096, 77, 40, "f16", 77, True),
        # One query a request over an encoder's states of up to 1000 rows: a step of a decoder that answers token by token.
        _encoder("encoder_16x16x1x64_states1000_f16", 16, 16, 16, 1, 1000, 64, "f16", 200, False),
        # The 64x64 level of the larger model's heads over the tokens of a reference image, ragged: the long case.
        _encoder("encoder_2x10x4096x64_states4173_bf16", 2, 10, 10, 4096, 4173, 64, "bf16", 3900, False),
        # Shared key/value heads of 128 over long prompts of up to 512 tokens, one of them empty.
        _encoder("encoder_8x16of4x1024x128_text512_bf16", 8, 16, 4, 1024, 512, 128, "bf16", 0, True),
        # Eight requests join or grow: the plan in front of every step.
        _plan("plan_8_page16", 8, 16, 0, 77, 1, 77),
        # A full server: 2048 requests with new tokens between one and 300.
        _plan("plan_2048_page64", 2048, 64, 0, 4000, 1, 300),
        # 64 prompts of up to 77 tokens enter the cache whole, 20 heads of 64.
        _write("write_64prompts_20x64_page16_f16", 64, 20, 64, 16, "f16", 0, 0, 20, 77),
        # One more token for each of 256 requests, into pages that other tokens share.
        _write("write_256tokens_8x128_page64_bf16", 256, 8, 128, 64, "bf16", 1, 900, 1, 1),
        # Few short requests, one query each: where latency counts.
        _cached("cached_4x8x1x64_len300_page16_f16", 4, 8, 8, 1, 1, 20, 300, 64, 16, "f16", False),
        # A full server's step: 64 requests of up to 8000 cached tokens, 32 heads over 8.
        _cached("cached_64x32of8x1x128_len8000_page64_bf16", 64, 32, 8, 1, 1, 300, 8000, 128, 64, "bf16", False),
        # Images of different sizes over text of 20 to 154 cached tokens, heads of 40.
        _cached("cached_8x8x4096x40_text154_page16_f16", 8, 8, 8, 1024, 4096, 20, 154, 40, 16, "f16", False),
        # The last 2048 tokens of two long sequences over all before them, causal, 16 heads over 4.
        _cached("cached_2x16of4x2048x128_len6000_page128_f16", 2, 16, 4, 2000, 2048, 5500, 6000, 128, 128, "f16", True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _flops(c):
    if c["kind"] == "encoder":
        return 4 * c["batch"] * c["heads"] * c["nq"] * c["nk"] * c["d"]
    return 4 * c["batch"] * c["heads"] * c["nq_hi"] * c["len_hi"] * c["d"]


def draw(rng):
    """One more case: any head size that is a multiple of 8 up to 160 (half the time one that models use), grouped heads,
    odd lengths."""
    kind = rng.choice(["encoder"] * 4 + ["plan"] + ["write"] * 2 + ["cached"] * 4)
    d = rng.choice([40, 64, 80, 128, 160]) if rng.random() < 0.5 else 8 * rng.randint(2, 20)
    dtype = rng.choice(["f16", "bf16"])
    page = rng.choice([16, 32, 64, 128])
    while True:
        kv_heads = rng.choice([1, 2, 4, 5, 8, 10, 16, 20])
        heads = kv_heads * rng.choice([1, 1, 1, 2, 4, 8])
        if kind == "encoder":
            nk = _log_int(rng, 1, 4500)
            nq = 1 if rng.random() < 0.2 else _log_int(rng, 1, 4500)
            c = _encoder("", _log_int(rng, 1, 32), heads, kv_heads, nq, nk, d, dtype, nk if rng.random() < 0.4 else rng.randint(0, nk),
                         rng.random() < 0.5)
            B = c["batch"]
            ok = _flops(c) <= 8e10 and B * heads * nq * nk <= 3e8 and B * (heads * nq + 2 * kv_heads * nk) * d <= 6e7
        elif kind == "plan":
            hi, new = _log_int(rng, 1, 4000), _log_int(rng, 1, 300)
            c = _plan("", _log_int(rng, 1, 2048), page, rng.randint(0, hi), hi, rng.randint(0, new), new)
            ok = True
        elif kind == "write":
            grown = rng.random() < 0.6
            hi = _log_int(rng, 1, 900) if grown else 0
            new = _log_int(rng, 1, 300)
            c = _write("", _log_int(rng, 1, 256), kv_heads, d, page, dtype, rng.randint(0, hi), hi, rng.randint(1, new), new)
            ok = c["batch"] * (hi + new) * kv_heads * d <= 6e7
        else:
            hi = _log_int(rng, 1, 8000)
            nq = 1 if rng.random() < 0.4 else _log_int(rng, 1, 4096)
            causal = rng.random() < 0.4 and nq <= hi
            c = _cached("", _log_int(rng, 1, 64), heads, kv_heads, rng.randint(1, nq), nq, rng.randint(nq if causal else 0, hi), hi, d, page, dtype,
                        causal)
            B = c["batch"]
            ok = _flops(c) <= 8e10 and B * heads * nq * hi <= 3e8 and B * heads * nq * d <= 5e7 and B * kv_heads * hi * d <= 4e8
        if ok:
            del c["name"]
            return c


# ------------------------------------------------------------------------------------------ inputs
def _spread(lo, hi, n):
    return np.rint(np.linspace(lo, hi, n)).astype(np.int64) if n > 1 else np.array([hi], dtype=np.int64)


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dtype)


def _starts(n):
    return np.concatenate([[0], np.cumsum(n)])


def _paged(order, lens, page, spare, max_pages):
    """Block table [B, max_pages] with the pages of `lens` tokens in a random order, the pages that are left, their number."""
    need = -(-lens // page)
    total = int(need.sum())
    pages = order.permutation(total + spare)
    table = np.full((len(lens), max_pages), -1, dtype=np.int64)
    table[np.arange(max_pages)[None, :] < need[:, None]] = pages[:total]
    return table, pages[total:], total + spare


def _codes(gen, n_pages, heads, page, d):
    """Codes and scales of a cache whose rows were normal: the largest of a page's values lies at about four deviations."""
    width = -(-d // 16) * 16
    c = torch.zeros(n_pages, heads, page, width, dtype=torch.int8, device="cuda")
    c[..., :d] = torch.randn(n_pages, heads, page, d, generator=gen, device="cuda", dtype=torch.float16).mul_(32).round_().clamp_(-127, 127)
    s = torch.randn(n_pages, heads, generator=gen, device="cuda").mul_(0.2).exp_().mul_(4.0 / 127.0)
    return c, s


class _Cache:
    """The buffers of a cache: codes [pages, kv heads, page, row] (rows of d codes, padded to a multiple of 16 with zeros)
    and scales [pages, kv heads]."""

    def __init__(self, gen, n_pages, heads, page, d):
        self.page, self.d = page, d
        self.k, self.k_scale = _codes(gen, n_pages, heads, page, d)
        self.v, self.v_scale = _codes(gen, n_pages, heads, page, d)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    order = np.random.RandomState(int(seed) % (2 ** 32))
    kind, B = case["kind"], case["batch"]
    s = dict(kind=kind)
    if kind == "encoder":
        H, G, nq, nk, d = (case[k] for k in ("heads", "kv_heads", "nq", "nk", "d"))
        t = _TYPES[case["dtype"]]
        s["q"] = torch.randn(B, nq, H, d, generator=gen, device="cuda").to(t)
        if case["fused"]:
            kv = torch.randn(B, nk, 2, G, d, generator=gen, device="cuda").to(t)
            s["k"], s["v"] = kv[:, :, 0], kv[:, :, 1]
        else:
            s["k"], s["v"] = (torch.randn(B, nk, G, d, generator=gen, device="cuda").to(t) for _ in range(2))
        s["lens"] = None if case["lo"] == nk else _dev(order.permutation(_spread(case["lo"], nk, B)))
    elif kind == "plan":
        page = case["page"]
        lens, new = (order.permutation(_spread(case[k + "_lo"], case[k + "_hi"], B)) for k in ("len", "new"))
        max_pages = -(-(case["len_hi"] + case["new_hi"]) // page)
        table, free, _ = _paged(order, lens, page, B * max_pages, max_pages)
        # room for the tokens in steps of 64, as a program with captured graphs has it
        s.update(page=page, lens=_dev(lens), new=_dev(new), table=_dev(table), free=_dev(free), n_tokens=max(64, -(-int(new.sum()) // 64) * 64))
    elif kind == "write":
        page, G, d = case["page"], case["kv_heads"], case["d"]
        t = _TYPES[case["dtype"]]
        lens, new = (order.permutation(_spread(case[k + "_lo"], case[k + "_hi"], B)) for k in ("len", "new"))
        total = lens + new
        table, _, n_pages = _paged(order, total, page, 4, int(-(-total.max() // page)))
        who = np.repeat(np.arange(B), new)
        at = lens[who] + np.arange(int(new.sum())) - _starts(new)[who]
        # what is read back: every row of the pages that were written
        first = lens // page * page
        kept = total - first
        back = np.repeat(np.arange(B), kept)
        row = first[back] + np.arange(int(kept.sum())) - _starts(kept)[back]
        T = len(who)
        s.update(cache=_Cache(gen, n_pages, G, page, d), slots=_dev(table[who, at // page] * page + at % page),
                 back=_dev(table[back, row // page] * page + row % page), type=t)
        s["k"], s["v"] = (torch.randn(T, G, d, generator=gen, device="cuda").to(t) for _ in range(2))
    else:
        H, G, d, page = (case[k] for k in ("heads", "kv_heads", "d", "page"))
        lens = order.permutation(_spread(case["len_lo"], case["len_hi"], B))
        nq = order.permutation(_spread(case["nq_lo"], case["nq_hi"], B))
        table, _, n_pages = _paged(order, lens, page, 4, max(1, -(-case["len_hi"] // page)))
        uniform = case["nq_lo"] == case["nq_hi"]
        q = torch.randn(int(nq.sum()), H, d, generator=gen, device="cuda").to(_TYPES[case["dtype"]])
        s.update(cache=_Cache(gen, n_pages, G, page, d), table=_dev(table), lens=_dev(lens), max_nq=case["nq_hi"], causal=case["causal"],
                 q=q.view(B, case["nq_hi"], H, d) if uniform else q, q_start=None if uniform else _dev(_starts(nq)))
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _attend(q, k, v, seen):
    """q [B, nq, H, d], k and v [B, nk, G, d] in 32 bits, seen [B, nq or 1, nk]: softmax(q k^T / sqrt(d)) v over the keys that
    a row sees, zeros for a row that sees none."""
    B, nq, H, d = q.shape
    G = k.shape[2]
    t = torch.matmul((q * (1.0 / math.sqrt(d))).view(B, nq, G, H // G, d).permute(0, 2, 3, 1, 4).reshape(B, G, H // G * nq, d), k.permute(0, 2, 3, 1))
    t = t.view(B, G, H // G, nq, -1).masked_fill_(~seen[:, None, None], float("-inf"))
    top = t.amax(-1, keepdim=True)
    t = t.sub_(torch.where(top == float("-inf"), 0.0, top)).exp_()
    total = t.sum(-1, keepdim=True)
    v = v.masked_fill(~seen.any(1)[:, :, None, None], 0.0)
    o = torch.matmul(t.view(B, G, H // G * nq, -1), v.permute(0, 2, 1, 3)).view(B, G, H // G, nq, d)
    o = torch.where(total > 0, o / total, 0.0)
    return o.permute(0, 3, 1, 2, 4).reshape(B, nq, H, d)


def _plain_encoder(s):
    q, k, v, lens = s["q"], s["k"], s["v"], s["lens"]
    at = torch.arange(k.shape[1], device="cuda")
    n = lens[:, None, None] if lens is not None else torch.full((q.shape[0], 1, 1), k.shape[1], device="cuda")
    return _attend(q.float(), k.float(), v.float(), at[None, None, :] < n).to(q.dtype)


def _plain_plan(s):
    lens, new, table, free, page = s["lens"].long(), s["new"].long(), s["table"], s["free"], s["page"]
    zero = torch.zeros(1, dtype=torch.int64, device="cuda")
    start = torch.cat([zero, new.cumsum(0)])
    have, need = (lens + page - 1) // page, (lens + new + page - 1) // page
    taken = (need - have).cumsum(0)
    col = torch.arange(table.shape[1], device="cuda")[None, :]
    at = (taken - (need - have))[:, None] + col - have[:, None]
    table = torch.where((col >= have[:, None]) & (col < need[:, None]), free[at.clamp(0, free.numel() - 1)], table)
    t = torch.arange(s["n_tokens"], device="cuda")
    who = (torch.searchsorted(start, t, right=True) - 1).clamp(max=lens.numel() - 1)
    pos = (lens[who] + t - start[who]).clamp(min=0)
    slot = table[who, (pos // page).clamp(max=table.shape[1] - 1)] * page + pos % page
    slots = torch.where(t < start[-1], slot, -1)
    return dict(table=table, start=start.int(), lens=(lens + new).int(), slots=slots.int(), used=taken[-1:].int())


def _plain_quantize(x, slots, codes, scale, page, d):
    """New codes and scales after the rows x [T, G, d] have entered the slots: a page that gets its first row takes its scale from
    the rows that come, a page that holds rows keeps the larger one and has its codes rounded to it."""
    P, G = scale.shape
    where, row = (slots // page).long(), (slots % page).long()
    x = x.float()
    top = torch.zeros(P, G, device="cuda").index_reduce_(0, where, x.abs().amax(-1), "amax")
    first = torch.full((P,), page, device="cuda").index_reduce_(0, where, row, "amin")
    touched, held = first < page, (first < page) & (first > 0)
    s = top * (1.0 / 127.0)
    s = torch.where(held[:, None], torch.maximum(s, scale), s)
    s = torch.where(touched[:, None], s, scale)
    old = codes[..., :d].float() * scale[..., None, None] / s[..., None, None]
    old = torch.where((s > scale)[..., None, None], old.round().clamp(-127, 127), codes[..., :d].float())
    mine = held[:, None] & (torch.arange(page, device="cuda")[None, :] < first[:, None])
    codes = codes.clone()
    codes[..., :d] = torch.where(mine[:, None, :, None], old, codes[..., :d].float()).to(torch.int8)
    q = torch.where(s[where][..., None] > 0, x / s[where][..., None], 0.0).round().clamp(-127, 127)
    codes.permute(0, 2, 1, 3)[where, row] = torch.nn.functional.pad(q, (0, codes.shape[3] - d)).to(torch.int8)
    return codes, s


def _plain_values(codes, scale, slots, page, d):
    where, row = (slots // page).long(), (slots % page).long()
    return codes.permute(0, 2, 1, 3)[where, row][..., :d].float() * scale[where][..., None]


def _plain_write(s):
    c = s["cache"]
    k, ks = _plain_quantize(s["k"], s["slots"], c.k, c.k_scale, c.page, c.d)
    v, vs = _plain_quantize(s["v"], s["slots"], c.v, c.v_scale, c.page, c.d)
    return dict(k=_plain_values(k, ks, s["back"], c.page, c.d).to(s["type"]), v=_plain_values(v, vs, s["back"], c.page, c.d).to(s["type"]),
                k_scale=ks, v_scale=vs)


def _plain_cached(s):
    c, table, lens, q = s["cache"], s["table"], s["lens"].long(), s["q"]
    B = table.shape[0]
    at = torch.arange(table.shape[1] * c.page, device="cuda")
    pages = table.long().clamp(min=0)
    k, v = ((codes[pages][..., :c.d].float() * scale[pages][..., None, None]).permute(0, 1, 3, 2, 4).reshape(B, at.numel(), -1, c.d)
            for codes, scale in ((c.k, c.k_scale), (c.v, c.v_scale)))
    i = torch.arange(s["max_nq"], device="cuda")[None, :]
    if s["q_start"] is None:
        n, x = torch.full((B, 1), s["max_nq"], device="cuda"), q
    else:
        start = s["q_start"].long()
        n = (start[1:] - start[:-1])[:, None]
        x = q[(start[:-1, None] + i).clamp(max=q.shape[0] - 1)]
    sees = (lens[:, None] - n + i + 1).clamp(min=0) if s["causal"] else lens[:, None].expand(B, s["max_nq"])
    o = _attend(x.float(), k, v, at[None, None, :] < sees[:, :, None]).to(q.dtype)
    return o if s["q_start"] is None else o[i < n]


def run(state):
    s = state
    kind = s["kind"]
    if own:
        from paper_2501_04304_b200 import binding as b
        if kind == "encoder":
            return b.encoder_attn(s["q"], s["k"], s["v"], kv_lens=s["lens"])
        if kind == "plan":
            start, lens, slots, used = b.kv_plan(s["lens"], s["new"], s["free"], s["table"], s["page"], s["n_tokens"])
            return dict(table=s["table"], start=start, lens=lens, slots=slots, used=used)
        c = s["cache"]
        cache = b.KvCache(c.k, c.v, c.k_scale, c.v_scale, c.d)
        if kind == "write":
            b.kv_write(cache, s["k"], s["v"], s["slots"])
            k, v = b.kv_read(cache, s["back"], s["type"])
            return dict(k=k, v=v, k_scale=c.k_scale, v_scale=c.v_scale)
        return b.cached_attn(s["q"], cache, s["table"], s["lens"], q_start=s["q_start"], max_nq=s["max_nq"], causal=s["causal"])
    return dict(encoder=_plain_encoder, plan=_plain_plan, write=_plain_write, cached=_plain_cached)[kind](s)


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    kind, B = case["kind"], case["batch"]
    if kind == "plan":
        lens, new = _spread(case["len_lo"], case["len_hi"], B), _spread(case["new_lo"], case["new_hi"], B)
        pages = int((lens + new).sum()) // case["page"] + B
        return {"bytes": 4 * (4 * B + 2 * pages + int(new.sum())), "flops": 0}
    if kind == "write":
        page, row = case["page"], case["kv_heads"] * case["d"]
        lens, new = _spread(case["len_lo"], case["len_hi"], B), _spread(case["new_lo"], case["new_hi"], B)
        kept = int((lens % page + new).sum())
        # rows in (16 bits), codes written, values out; a scale for each page and head
        return {"bytes": 2 * row * (3 * int(new.sum()) + 2 * kept) + 8 * case["kv_heads"] * (kept // page + B), "flops": 6 * row * int(new.sum())}
    d, H, G = case["d"], case["heads"], case["kv_heads"]
    if kind == "encoder":
        lens = _spread(case["lo"], case["nk"], B)
        n, pairs = B * case["nq"], int(lens.sum()) * case["nq"]
        return {"bytes": 4 * n * H * d + 4 * int(lens.sum()) * G * d, "flops": 4 * pairs * H * d}
    lens, nq = _spread(case["len_lo"], case["len_hi"], B), _spread(case["nq_lo"], case["nq_hi"], B)
    pairs = float(nq.mean() * lens.sum()) - (float((nq * (nq - 1)).sum()) / 2 if case["causal"] else 0.0)
    scales = 8 * G * int((-(-lens // case["page"])).sum())
    return {"bytes": 4 * int(nq.sum()) * H * d + 2 * int(lens.sum()) * G * d + scales, "flops": 4 * pairs * H * d}


# ------------------------------------------------------------------------------------------ 64 bits
def _exact_rows(q, k, v, sees):
    """q [n, H, d], k and v [m, G, d] in 64 bits, row i sees the first sees[i] keys."""
    n, H, d = q.shape
    o = torch.zeros(n, H, d, dtype=torch.float64, device="cuda")
    if not k.shape[0]:
        return o
    hidden = torch.arange(k.shape[0], device="cuda")[None, :] >= sees[:, None]
    some = sees > 0
    for h in range(H):
        g = h // (H // k.shape[1])
        t = (q[:, h] @ k[:, g].T / math.sqrt(d)).masked_fill(hidden, float("-inf"))
        o[some, h] = torch.softmax(t[some], -1) @ v[:, g]
    return o


def _exact_cache(x, slots, codes, scale, page, d):
    codes, scale = codes[..., :d].double(), scale.double()
    by_page = {}
    for t, slot in enumerate(slots.tolist()):
        by_page.setdefault(slot // page, []).append((slot % page, t))
    for p, rows in by_page.items():
        at = torch.tensor([r for r, _ in rows], device="cuda")
        new = x[torch.tensor([t for _, t in rows], device="cuda")].double()
        first = int(at.min())
        s = new.abs().amax((0, 2)) / 127
        if first:
            s = torch.maximum(s, scale[p])
            grown = (s > scale[p])[:, None, None]
            codes[p, :, :first] = torch.where(grown, torch.round(codes[p, :, :first] * (scale[p] / s)[:, None, None]), codes[p, :, :first])
        codes[p][:, at] = torch.round(new / s[None, :, None]).transpose(0, 1)
        scale[p] = s
    return codes * scale[..., None, None], scale


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "plan":
        return None
    if kind == "encoder":
        B, nk = case["batch"], case["nk"]
        lens = [nk] * B if s["lens"] is None else s["lens"].tolist()
        return torch.stack([_exact_rows(s["q"][b].double(), s["k"][b, :n].double(), s["v"][b, :n].double(),
                                        torch.full((case["nq"],), n, device="cuda")) for b, n in enumerate(lens)])
    c = s["cache"]
    if kind == "write":
        out = {}
        for name, x, codes, scale in (("k", s["k"], c.k, c.k_scale), ("v", s["v"], c.v, c.v_scale)):
            values, out[name + "_scale"] = _exact_cache(x, s["slots"], codes, scale, c.page, c.d)
            back = s["back"].long()
            out[name] = values[back // c.page, :, back % c.page]
        return out
    B, H, d = case["batch"], case["heads"], case["d"]
    q = s["q"].reshape(-1, H, d)
    starts = [b * s["max_nq"] for b in range(B + 1)] if s["q_start"] is None else s["q_start"].tolist()
    rows = []
    for b, n in enumerate(s["lens"].tolist()):
        pages = s["table"][b, :-(-n // c.page)].long()
        k, v = ((codes[pages][..., :d].double() * scale[pages].double()[..., None, None]).transpose(1, 2).reshape(-1, case["kv_heads"], d)[:n]
                for codes, scale in ((c.k, c.k_scale), (c.v, c.v_scale)))
        nq = starts[b + 1] - starts[b]
        sees = torch.full((nq,), n, device="cuda")
        if case["causal"]:
            sees = (n - nq + 1 + torch.arange(nq, device="cuda")).clamp(min=0)
        rows.append(_exact_rows(q[starts[b]:starts[b + 1]].double(), k, v, sees))
    return torch.cat(rows).reshape(s["q"].shape)
