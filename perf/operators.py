"""The operators of the paged key/value cache: appending with the rotary encoding on the way (esa_append_paged) and the attention that
reads the cache (esa_attend_paged), scores capped by a tanh among them.

A case is a ragged batch of sequences over one pool of pages.  `run` computes it with the framework's calls where `own` is true and with
elementary torch operations where it is not; `exact` is the definition in 64 bits, sequence by sequence.
"""
import math
import random

import torch

own = False

F8_MAX = 448.0                  # the largest e4m3 number
LOW, HIGH = 27, 239             # exponents of a block: 2^(byte - 127)
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------- the cases
def _append(name, n_seq, new, ctx, h, h_kv, d, page, dtype, held, ragged):
    return dict(name=name, op="append", n_seq=n_seq, new=new, ctx=ctx, h=h, h_kv=h_kv, d=d, page=page, dtype=dtype, held=held, ragged=ragged,
                mix=1, view="all", l_i=0, l_l=0, n_sel=0, cap=0.0)


def _attend(name, n_seq, new, ctx, h, h_kv, d, page, dtype, held, ragged, view="all", l_i=0, l_l=0, n_sel=0, cap=0.0):
    return dict(name=name, op="attend", n_seq=n_seq, new=new, ctx=ctx, h=h, h_kv=h_kv, d=d, page=page, dtype=dtype, held=held, ragged=ragged,
                mix=1, view=view, l_i=l_i, l_l=l_l, n_sel=n_sel, cap=cap)


def listed():
    return [
        # a decode step of sixteen conversations of different lengths: latency
        _append("append_decode_16", 16, 1, 262144, 32, 8, 128, 64, "bf16", "e4m3", True),
        # prompts of different lengths taken in at once: bandwidth, and the largest of the appends
        _append("append_prompts_8", 8, 4096, 8192, 32, 8, 128, 64, "bf16", "e4m3", True),
        # short fp32 chunks, pages in the storage type, a head for every query head
        _append("append_f32_pages", 4, 100, 1000, 8, 8, 64, 16, "f32", "same", True),
        # the first tokens of one conversation: the smallest attention, latency
        _attend("attend_one_short", 1, 1, 301, 32, 8, 128, 64, "bf16", "e4m3", False),
        # one long document read token by token: the whole cache for every token
        _attend("attend_decode_256k", 1, 1, 262144, 32, 8, 128, 64, "bf16", "e4m3", False),
        # a decode step of sixteen conversations of different lengths over 8-bit pages
        _attend("attend_decode_16", 16, 1, 65536, 32, 8, 128, 64, "bf16", "e4m3", True),
        # ESA's chunk: 512 tokens see 128 initial, 2048 selected, 2048 local ones of 128 thousand, and themselves
        _attend("attend_esa_chunk", 1, 512, 131072, 32, 8, 128, 64, "bf16", "e4m3", False, "esa", 128, 2048, 2048),
        # ESA's decode step of sixteen conversations, bf16 pages
        _attend("attend_esa_decode_16", 16, 1, 32768, 32, 8, 128, 32, "bf16", "same", True, "esa", 128, 2048, 2048),
        # chunks of prompts over what came before them, everything visible: the most arithmetic
        _attend("attend_prompts_4", 4, 1024, 16384, 32, 8, 128, 64, "bf16", "e4m3", True),
        # fp32 with drafted tokens, two KV heads
        _attend("attend_f32_drafts", 3, 5, 3000, 16, 2, 64, 16, "f32", "same", True),
        # capped scores: a decode step, and a chunk over bf16 pages of head size 64
        _attend("attend_cap_decode_8", 8, 1, 8192, 32, 8, 128, 64, "bf16", "e4m3", True, cap=30.0),
        _attend("attend_cap_chunk", 2, 333, 5000, 32, 8, 64, 64, "bf16", "same", True, cap=50.0),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    h, h_kv = rng.choice(((32, 8), (16, 2), (8, 8), (4, 1)))
    d, page = rng.choice((64, 128)), rng.choice((16, 32, 64, 128))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    held = rng.choice(("e4m3", "e4m3", "same"))
    if rng.random() < 0.33:
        n_seq, new = spread(1, 16), spread(1, 1024)
        return dict(op="append", n_seq=n_seq, new=new, ctx=new + spread(1, 100000), h=h, h_kv=h_kv, d=d, page=page, dtype=dtype, held=held,
                    ragged=True, mix=rng.randrange(1 << 20), view="all", l_i=0, l_l=0, n_sel=0, cap=0.0)
    cap = rng.choice((0.0, 0.0, 30.0, 50.0))
    view = rng.choice(("all", "esa"))
    if rng.random() < 0.6:                                        # a step of few tokens
        n_seq, new = spread(1, 16), spread(1, 8)
        ctx = new + spread(1, 400000 // n_seq)
    else:                                                         # a chunk
        n_seq, new = spread(1, 3), spread(17, 700)
        ctx = new + spread(1, 8000)
    if dtype == "f32":
        ctx = new + min(ctx - new, 30000 // n_seq)
    l_i, l_l, n_sel = (rng.randrange(200), spread(1, 2500), spread(1, 2500)) if view == "esa" else (0, 0, 0)
    return dict(op="attend", n_seq=n_seq, new=new, ctx=ctx, h=h, h_kv=h_kv, d=d, page=page, dtype=dtype, held=held, ragged=True,
                mix=rng.randrange(1 << 20), view=view, l_i=l_i, l_l=l_l, n_sel=n_sel, cap=cap)


def _lengths(case):
    """(tokens before the call, new tokens) of every sequence; the first one has the case's own."""
    r = random.Random(case["mix"])
    start, new = [], []
    for b in range(case["n_seq"]):
        n = case["new"] if b == 0 or not case["ragged"] else r.randint(max(1, case["new"] // 4), case["new"])
        total = case["ctx"] if b == 0 or not case["ragged"] else max(n, r.randint(case["ctx"] // 4, case["ctx"]))
        start.append(total - n)
        new.append(n)
    return start, new


def _segments(t0, case):
    if case["view"] == "all":
        return t0, t0
    i_end = min(case["l_i"], t0)
    return i_end, max(t0 - case["l_l"], i_end)


def work(case):
    es, cs = (2 if case["dtype"] == "bf16" else 4), (1 if case["held"] == "e4m3" else 2 if case["dtype"] == "bf16" else 4)
    h, h_kv, d = case["h"], case["h_kv"], case["d"]
    start, new = _lengths(case)
    if case["op"] == "append":
        n = sum(new)
        return {"bytes": n * d * ((2 * h + 2 * h_kv) * es + 2 * h_kv * cs), "flops": n * d * 3 * (h + h_kv)}
    rows = pairs = 0
    for t0, n in zip(start, new):
        i_end, l_start = _segments(t0, case)
        seen = i_end + min(case["n_sel"], l_start - i_end) + t0 - l_start
        rows += seen + n
        pairs += seen * n + n * (n + 1) // 2
    return {"bytes": rows * h_kv * d * 2 * cs + sum(new) * h * d * 2 * es, "flops": 4 * h * d * pairs}


# ---------------------------------------------------------------- blocks in 8 bits
def _exponent(amax):
    """The byte of the smallest power of two s with amax <= 448 s, within [LOW, HIGH]."""
    m, e = torch.frexp(amax.float())                              # amax = m 2^e, m in [1/2, 1); 448 = 0.875 * 2^9
    return torch.where(amax > 0, e - torch.where(m <= 0.875, 9, 8) + 127, LOW).clamp(LOW, HIGH)


def _to_f8(x, byte):
    return torch.ldexp(x.float(), 127 - byte).clamp(-F8_MAX, F8_MAX).to(torch.float8_e4m3fn)


def _of_f8(values, byte):
    return torch.ldexp(values.float(), byte.int() - 127)


def _bytes(t):
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


# ---------------------------------------------------------------- what a program has in hand
def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt, P, h, h_kv, d, B = TYPES[case["dtype"]], case["page"], case["h"], case["h_kv"], case["d"], case["n_seq"]
    start, new = _lengths(case)
    s = dict(case=case, max_new=max(new), max_len=max(a + b for a, b in zip(start, new)), scale=1.0 / math.sqrt(d), base=5e5)
    s["start"] = torch.tensor(start, dtype=torch.int32, device=dev)
    s["cu"] = torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32, device=dev)
    n_tok, width = sum(new), -(-s["max_len"] // P)
    # an append's program is measured over the pages that it writes; those in front of them stand for one shared beginning
    first = [a // P if case["op"] == "append" else 0 for a in start]
    need = [-(-(a + n) // P) - f for a, n, f in zip(start, new, first)]
    n_pages = sum(need) + 4
    order = torch.randperm(n_pages - 1, generator=g, device=dev).to(torch.int32)
    table = torch.full((B, width), n_pages - 1, dtype=torch.int32, device=dev)
    for b in range(B):
        table[b, first[b]:first[b] + need[b]] = order[sum(need[:b]):sum(need[:b + 1])]
    s["pages"] = table

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32)

    s["q"] = normal(n_tok, h, d).to(dt)
    if case["op"] == "append":
        s["k"], s["v"] = normal(n_tok, h_kv, d).to(dt), normal(n_tok, h_kv, d).to(dt)
    # keys whose channels differ in size, values of unit size
    sizes = 1.5 * torch.rand((h_kv, 1, d), generator=g, device=dev) + 0.25
    for name, by in (("k", sizes), ("v", 1.0)):
        held = torch.empty((n_pages, h_kv, P, d), dtype=torch.float8_e4m3fn if case["held"] == "e4m3" else dt, device=dev)
        byte = torch.empty((n_pages, h_kv), dtype=torch.uint8, device=dev)
        part = max(1, (1 << 27) // (h_kv * P * d))
        for at in range(0, n_pages, part):
            x = (normal(*held[at:at + part].shape) * by).to(dt)
            if case["held"] == "e4m3":
                e = _exponent(x.abs().amax((2, 3)))
                byte[at:at + part] = e.to(torch.uint8)
                _bytes(held[at:at + part]).copy_(_bytes(_to_f8(x, e[:, :, None, None])))
            else:
                held[at:at + part] = x
        s[name + "_cache"], s[name + "_scale"] = held, byte if case["held"] == "e4m3" else None
    s["idx"] = None
    if case["view"] == "esa":
        idx = torch.full((B, case["n_sel"]), -1, dtype=torch.int32, device=dev)
        for b, t0 in enumerate(start):
            i_end, l_start = _segments(t0, case)
            k = min(case["n_sel"], l_start - i_end)
            if k:
                idx[b, :k] = (torch.randperm(l_start - i_end, generator=g, device=dev)[:k].sort().values + i_end).to(torch.int32)
        s["idx"] = idx
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if own:
        import paper_2502_14477_amd as esa
        if case["op"] == "append":
            q = esa.esa_append_paged(s["k"], s["v"], s["cu"], s["start"], s["pages"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"],
                                     q=s["q"], rope_base=s["base"])
            return _written(s, q)
        l_i, l_l = (None, 0) if case["view"] == "all" else (case["l_i"], case["l_l"])
        return esa.esa_attend_paged(s["q"], s["cu"], s["start"], s["pages"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"],
                                    l_i=l_i, l_l=l_l, idx=s["idx"], scale=s["scale"], cap=case["cap"])
    return _plain_append(s) if case["op"] == "append" else _plain_attend(s)


def _written(s, q):
    got = {"q": q, "k": s["k_cache"], "v": s["v_cache"]}
    if s["k_scale"] is not None:
        got.update(k_scale=s["k_scale"], v_scale=s["v_scale"])
    return got


def _turn(x, pos, base):
    """Rows [n, heads, d] turned to their positions, in 64 bits and rounded once."""
    half = x.shape[-1] // 2
    freq = base ** (-2.0 * torch.arange(half, dtype=torch.float64, device=x.device) / x.shape[-1])
    angle = pos.double()[:, None, None] * freq
    c, t = angle.cos(), angle.sin()
    a, b = x[..., :half].double(), x[..., half:].double()
    return torch.cat((a * c - b * t, b * c + a * t), -1).to(x.dtype)


def _plain_append(s):
    case, P = s["case"], s["case"]["page"]
    cu, start, pages = s["cu"].long(), s["start"].long(), s["pages"].long()
    n_tok = s["k"].shape[0]
    tok = torch.arange(n_tok, device=cu.device)
    b = torch.searchsorted(cu[1:].contiguous(), tok, right=True)
    pos = start[b] + tok - cu[b]
    q = _turn(s["q"], pos, s["base"])
    rows = {"k": _turn(s["k"], pos, s["base"]), "v": s["v"]}
    if case["held"] == "same":
        page, slot = pages[b, pos // P], pos % P
        for name in ("k", "v"):
            s[name + "_cache"][page, :, slot] = rows[name]
        return _written(s, q)
    # every page that a sequence writes to, whole: [B, pages of a sequence, h_kv, P, d]; a sequence with fewer pages repeats its first
    length = start + cu[1:] - cu[:-1]
    n = start[:, None] // P + torch.arange(s["max_new"] // P + 2, device=cu.device)
    n = torch.where(n * P < length[:, None], n, start[:, None] // P)
    page = pages.gather(1, n)
    at = n[:, :, None] * P + torch.arange(P, device=cu.device)
    fresh = (at >= start[:, None, None]) & (at < length[:, None, None])
    source = (cu[:-1, None, None] + at - start[:, None, None]).clamp(0, n_tok - 1)
    fresh = fresh[:, :, None, :, None]
    for name in ("k", "v"):
        cache, scale = s[name + "_cache"], s[name + "_scale"]
        old, old_byte = _bytes(cache)[page].view(torch.float8_e4m3fn).float(), scale[page].int()
        x = rows[name].float()[source].transpose(2, 3)            # [B, pages, h_kv, P, d]
        byte = _exponent(torch.where(fresh, x.abs(), 0.0).amax((3, 4)))
        byte = torch.where((n * P >= start[:, None])[:, :, None], byte, torch.maximum(byte, old_byte))
        behind = (at >= length[:, None, None])[:, :, None, :, None]
        kept = torch.where(behind, old, torch.ldexp(old, (old_byte - byte)[..., None, None]))
        held = torch.where(fresh, torch.ldexp(x, 127 - byte[..., None, None]).clamp(-F8_MAX, F8_MAX), kept).to(torch.float8_e4m3fn)
        _bytes(cache)[page] = _bytes(held)
        scale[page] = byte.to(torch.uint8)
    return _written(s, q)


def _positions(s):
    """Positions that a sequence's tokens may see [B, n], and whether each is there."""
    case, start = s["case"], s["start"].long()[:, None]
    length = start + (s["cu"][1:] - s["cu"][:-1]).long()[:, None]
    dev = start.device
    if case["view"] == "all":
        at = torch.arange(s["max_len"], device=dev).expand(start.shape[0], -1)
        return at, at < length
    i_end = start.clamp(max=case["l_i"])
    l_start = torch.maximum(start - case["l_l"], i_end)
    first = torch.arange(case["l_i"], device=dev).expand(start.shape[0], -1)
    chosen = s["idx"].long()
    late = l_start + torch.arange(case["l_l"] + s["max_new"], device=dev)
    there = torch.cat((first < i_end, (chosen >= i_end) & (chosen < l_start), late < length), 1)
    return torch.cat((first, chosen, late), 1), there


def _plain_attend(s):
    case, P = s["case"], s["case"]["page"]
    h, h_kv, d, B = case["h"], case["h_kv"], case["d"], case["n_seq"]
    cu, start, pages = s["cu"].long(), s["start"].long(), s["pages"].long()
    at, there = _positions(s)
    safe = torch.where(there, at, 0)
    page, slot = pages.gather(1, safe // P), safe % P

    def seen(name):                                               # [B, h_kv, n, d], 0 where nothing is
        x = _bytes(s[name + "_cache"])[page, :, slot]
        if case["held"] == "e4m3":
            x = _of_f8(x.view(torch.float8_e4m3fn), s[name + "_scale"][page][..., None])
        return torch.where(there[:, :, None, None], x.float(), 0.0).transpose(1, 2).contiguous()

    new = torch.arange(s["max_new"], device=cu.device)
    source = cu[:-1, None] + new                                  # a sequence's tokens, the last one's again where it has fewer
    source = torch.minimum(source, cu[1:, None] - 1)
    q = s["q"].float()[source].view(B, -1, h_kv, h // h_kv, d).transpose(1, 2).reshape(B, h_kv, -1, d)
    logits = torch.matmul(q, seen("k").transpose(2, 3).contiguous()) * s["scale"]
    if case["cap"] > 0:
        logits = case["cap"] * torch.tanh(logits / case["cap"])
    visible = there[:, None, :] & (at[:, None, :] <= (start[:, None] + new)[:, :, None])
    visible = visible[:, None, :, None, :].expand(-1, h_kv, -1, h // h_kv, -1).reshape(B, h_kv, -1, at.shape[1])
    logits = torch.where(visible, logits, float("-inf"))
    p = torch.exp(logits - logits.amax(-1, keepdim=True))
    o = torch.matmul(p / p.sum(-1, keepdim=True), seen("v"))
    o = o.view(B, h_kv, -1, h // h_kv, d).transpose(1, 2).reshape(B, -1, h, d)
    tok = torch.arange(s["q"].shape[0], device=cu.device)
    b = torch.searchsorted(cu[1:].contiguous(), tok, right=True)
    return o[b, tok - cu[b]].to(s["q"].dtype)


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    if case["op"] == "attend" and work(case)["flops"] > 2e11:
        return None
    s = prepare(case, seed)
    start, new = _lengths(case)
    h, h_kv, d, P = case["h"], case["h_kv"], case["d"], case["page"]
    table = s["pages"].cpu().tolist()
    at = 0
    if case["op"] == "append":
        half = d // 2

        def turned(x, p0):
            p = torch.arange(p0, p0 + x.shape[0], dtype=torch.float64, device=x.device)
            w = torch.exp(torch.arange(half, dtype=torch.float64, device=x.device) * (-2.0 / d * math.log(s["base"])))
            z = torch.complex(x[..., :half].double(), x[..., half:].double()) * torch.polar(torch.ones((), dtype=torch.float64, device=x.device), torch.outer(p, w))[:, None]
            return torch.cat((z.real, z.imag), -1)

        q = torch.cat([turned(s["q"][sum(new[:b]):sum(new[:b + 1])], start[b]) for b in range(case["n_seq"])])
        got = {"q": q}
        if case["held"] == "e4m3":
            return dict(got, k=None, v=None, k_scale=None, v_scale=None)
        for name in ("k", "v"):
            got[name] = s[name + "_cache"].double()
        for b, (p0, n) in enumerate(zip(start, new)):
            rows = {"k": turned(s["k"][at:at + n], p0), "v": s["v"][at:at + n].double()}
            for i in range(n):
                for name in ("k", "v"):
                    got[name][table[b][(p0 + i) // P], :, (p0 + i) % P] = rows[name][i]
            at += n
        return got
    out = torch.empty((sum(new), h, d), dtype=torch.float64, device="cuda")
    for b, (t0, n) in enumerate(zip(start, new)):
        i_end, l_start = _segments(t0, case)
        chosen = [] if s["idx"] is None else [p for p in s["idx"][b].tolist() if i_end <= p < l_start]
        where = torch.tensor(list(range(i_end)) + chosen + list(range(l_start, t0 + n)), device="cuda")
        page, slot = s["pages"][b].long()[where // P], where % P
        limit = torch.arange(t0, t0 + n, device="cuda")
        for g in range(h_kv):
            kv = []
            for name in ("k", "v"):
                x = _bytes(s[name + "_cache"])[page, g, slot]
                if case["held"] == "e4m3":
                    x = x.view(torch.float8_e4m3fn).double() * torch.pow(2.0, s[name + "_scale"][page, g].double() - 127.0)[:, None]
                kv.append(x.double())
            for i in range(g * (h // h_kv), (g + 1) * (h // h_kv)):
                z = s["q"][at:at + n, i].double() @ kv[0].T.contiguous() * s["scale"]
                if case["cap"] > 0:
                    z = case["cap"] * torch.tanh(z / case["cap"])
                z.masked_fill_(where[None, :] > limit[:, None], float("-inf"))
                out[at:at + n, i] = torch.softmax(z, -1) @ kv[1]
        at += n
    return out
