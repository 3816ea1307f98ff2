"""Operators of language models on packed tokens, as cases to time, with their plain forms and their values in 64 bits.

Tokens of several requests lie one behind the other (``cu`` holds where each request begins, and the end of the last).  A
case names an operator and its sizes:

* ``slots``   block tables, slot maps, positions and offsets of a step, built from request lengths;
* ``rope``    rotary positions of queries and keys, or the gradient's inverse rotation;
* ``prompt``  causal attention over packed prompts with grouped heads; ``train`` adds the backward pass;
* ``append``  keys and values to the pages of a cache in 4 bits, and the values that the cache then holds;
* ``cached``  attention of new tokens over that cache: one token a request, several, or the nodes of a token tree.

Head sizes 64 and 128, bf16 and the softmax scale 1/sqrt(d) are those of the rest of the library.  Queries, keys and values are
N(0,1).  The cache holds groups of 32 values: the smallest exponent e with max|x| <= 7 * 2^e, between -120 and 125, as a byte
e + 127, and codes of x / 2^e on 0, .5, 1, 1.5, 2, 3, 4, 6 (nearest, ties to the even code, sign in bit 3), element 2i in the low half of byte i.
"""
import math

import torch

own = False

DEV = "cuda"
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    case = lambda name, op, **more: dict(name=name, op=op, **more)  # noqa: E731
    return [
        # one decoding step of a small server: the smallest call, all launch and latency
        case("slots-decode", "slots", R=64, new=1, ctx=8000, page=64),
        # a step that mixes prompts' chunks and single tokens of many requests
        case("slots-mixed", "slots", R=1000, new=256, ctx=16384, page=16),
        # positions of one decoding step
        case("rope-decode", "rope", T=33, H=32, Hk=8, d=128, rot=128, pairs="half", inverse=False, far=8192),
        # the gradient of a long batch: neighbouring pairs in half of each head, far positions with scaled frequencies
        case("rope-train", "rope", T=16381, H=32, Hk=8, d=128, rot=64, pairs="even", inverse=True, far=131072),
        # two long prompts, one of a length that no tile divides: the largest forward
        case("prompt-long", "prompt", R=2, L=8192, short=0, H=32, Hk=8, d=128),
        # many short prompts of uneven lengths
        case("prompt-short", "prompt", R=37, L=300, short=1, H=16, Hk=4, d=64),
        # fine-tuning on packed sequences: as many key heads as query heads, lengths down to a single token
        case("train-packed", "train", R=13, L=1024, short=1, H=16, Hk=16, d=64),
        # training on long sequences with grouped heads
        case("train-long", "train", R=2, L=4096, short=0, H=32, Hk=8, d=128),
        # the new tokens of a decoding step go into the cache
        case("append-decode", "append", T=64, Hk=8, d=128, page=64, pages=4096),
        # a prompt goes into the cache
        case("append-prompt", "append", T=16384, Hk=8, d=128, page=16, pages=8192),
        # decoding: one token of each request over a long cache
        case("cached-decode", "cached", R=64, new=1, L=16384, H=32, Hk=8, d=128, page=64, tree=False),
        # verification of a token tree of 256 nodes behind a prefix
        case("cached-tree", "cached", R=8, new=256, L=1280, H=32, Hk=32, d=128, page=32, tree=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["slots", "rope", "prompt", "train", "append", "cached", "cached"])
    d = rng.choice([64, 128])
    Hk = rng.choice([1, 2, 4, 8])
    H = Hk * rng.choice([1, 2, 3, 4, 8])
    if op == "slots":
        return dict(op=op, R=_log(rng, 1, 1000), new=_log(rng, 1, 256), ctx=_log(rng, 1, 16384), page=rng.choice([16, 32, 64, 128]))
    if op == "rope":
        return dict(op=op, T=_log(rng, 1, 16381), H=H, Hk=Hk, d=d, rot=rng.choice([d, d // 2, 2 * rng.randint(1, d // 2)]), pairs=rng.choice(["half", "even"]),
                    inverse=rng.random() < 0.5, far=_log(rng, 64, 1 << 20))
    if op in ("prompt", "train"):
        L = _log(rng, 1, 8192 if op == "prompt" else 4096)
        most = (1 << 31 if op == "prompt" else 1 << 30) // (L * L * H)
        return dict(op=op, R=_log(rng, 1, max(1, min(64, most, 32768 // L))), L=L, short=rng.choice([0, 1]), H=H, Hk=Hk, d=d)
    page = rng.choice([16, 32, 64, 128])
    if op == "append":
        T = _log(rng, 1, 16384)
        return dict(op=op, T=T, Hk=Hk, d=d, page=page, pages=-(-T // page) + _log(rng, 1, 4096))
    L, new = _log(rng, 1, 32768), rng.choice([1, 1, 1, 2, _log(rng, 1, 128)])
    R = _log(rng, 1, max(1, min(128, (1 << 20) // L, (1 << 31) // (H * new * L))))
    return dict(op=op, R=R, new=new, L=max(L, new), H=H, Hk=Hk, d=d, page=page, tree=new > 1 and rng.random() < 0.5)


def _lengths(case):
    """Lengths of a case's requests, the same ones for every seed: one of L, the others nearly as long or down to one token."""
    R, L = case["R"], case["L"]
    u = (torch.arange(R - 1, dtype=torch.float64) + 0.5) / max(1, R - 1)
    n = torch.exp(u * math.log(L)) if case["short"] else L * (0.6 + 0.4 * u)
    return torch.cat([torch.tensor([L]), n.round().clamp(1, L).to(torch.int64)])


def _step_lengths(case):
    """New tokens of each request of a step: one, or none to the most that there are."""
    R, new = case["R"], case["new"]
    return torch.ones(R, dtype=torch.int64) if new == 1 else torch.arange(R) * 7919 % (new + 1)


def _offsets(n):
    return torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(torch.int32).to(DEV)


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _fill_cache(g, pages, Hk, page, d):
    """Pages as a program finds them: codes and scales of N(0,1) data, in the layout of the cache."""
    codes = lambda: torch.randint(0, 256, (pages, Hk, page, d // 2), generator=g, device=DEV, dtype=torch.uint8)  # noqa: E731
    exps = lambda *s: torch.randint(125, 128, s, generator=g, device=DEV, dtype=torch.uint8)  # noqa: E731
    return {"k": codes(), "k_scale": exps(pages, Hk, page, d // 32), "v": codes(), "v_scale": exps(pages, Hk, d // 32, page)}


def _tree_bits(R, new, seed):
    """Which of its request's new tokens each node of a random tree sees, itself and its ancestors, as words of 64 bits."""
    g = torch.Generator().manual_seed(seed)
    parent = (torch.rand(R, new, generator=g) * torch.arange(new)).long()
    sees = torch.eye(new, dtype=torch.bool).expand(R, new, new).clone()
    rows = torch.arange(R)
    for i in range(1, new):
        sees[:, i] |= sees[rows, parent[:, i]]
    words = -(-new // 64)
    bits = torch.zeros(R, new, words * 64, dtype=torch.bool)
    bits[:, :, :new] = sees
    weight = torch.ones(64, dtype=torch.int64) << torch.arange(64)
    return (bits.view(R * new, words, 64).to(torch.int64) * weight).sum(-1).to(DEV)


def prepare(case, seed):
    op = case["op"]
    h = torch.Generator().manual_seed(seed * 7919 + 11)
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 12)
    s = dict(case, seed=seed)
    if op == "slots":
        R, page = case["R"], case["page"]
        ctx = torch.randint(0, case["ctx"] + 1, (R,), generator=h)
        new = _step_lengths(case)[torch.randperm(R, generator=h)]
        width = -(-(case["ctx"] + case["new"]) // page)
        held, want = -(-ctx // page), -(-(ctx + new) // page)
        ids = torch.randperm(int(want.sum()) + 17, generator=h).to(torch.int32)
        table = torch.full((R, width), -1, dtype=torch.int32)
        table[torch.arange(width) < held[:, None]] = ids[:int(held.sum())]
        T = int(new.sum()) + 5                                         # rows of the step's buffers, some behind the last token
        s |= dict(ctx_lens=ctx.to(torch.int32).to(DEV), new_lens=new.to(torch.int32).to(DEV), table=table.to(DEV), T=T,
                  free=ids.to(DEV), free_at=torch.tensor([int(held.sum())], dtype=torch.int32, device=DEV))
    elif op == "rope":
        T, H, Hk, d, rot = (case[x] for x in ("T", "H", "Hk", "d", "rot"))
        fused = _normal(g, T, (H + 2 * Hk) * d)                          # one projection's output: q, k and v side by side
        j = torch.arange(rot // 2, dtype=torch.float64)
        stretch = 1 + 3 * (j / max(1, rot // 2 - 1)).clamp(0.25, 0.75)   # slow pairs are slowed further in a longer context
        s |= dict(q=fused[:, :H * d].view(T, H, d), k=fused[:, H * d:(H + Hk) * d].view(T, Hk, d), mscale=1.0 if case["far"] <= 8192 else 1.125,
                  freqs=(10000.0 ** (-2 * j / rot) / (stretch if case["far"] > 8192 else 1)).to(torch.float32).to(DEV),
                  positions=torch.randint(0, case["far"], (T,), generator=g, device=DEV, dtype=torch.int32))
    elif op in ("prompt", "train"):
        n = _lengths(case)
        n = n[torch.randperm(len(n), generator=h)]
        T, H, Hk, d = int(n.sum()), case["H"], case["Hk"], case["d"]
        s |= dict(cu=_offsets(n), T=T, q=_normal(g, T, H, d), k=_normal(g, T, Hk, d), v=_normal(g, T, Hk, d))
        if op == "train":
            s["d_o"] = _normal(g, T, H, d)
    elif op == "append":
        T, Hk, d, page, pages = (case[x] for x in ("T", "Hk", "d", "page", "pages"))
        shape = torch.exp2(torch.randint(-3, 4, (T, Hk, 1), generator=g, device=DEV).float())
        s |= dict(k=(_normal(g, T, Hk, d).float() * shape).to(torch.bfloat16), v=_normal(g, T, Hk, d), cache=_fill_cache(g, pages, Hk, page, d),
                  slots=torch.randperm(pages * page, generator=g, device=DEV)[:T].to(torch.int32))
        if T > 8:
            s["slots"][-3:] = -1                                         # rows of a padded step
    else:
        R, new, H, Hk, d, page, L = (case[x] for x in ("R", "new", "H", "Hk", "d", "page", "L"))
        lens = (L * (0.5 + 0.5 * torch.rand(R, generator=h))).round().to(torch.int64).clamp(new, L)
        lens[0] = L
        width = -(-L // page)
        pages = R * width + 3
        table = torch.randperm(pages, generator=h)[:R * width].view(R, width).to(torch.int32)
        s |= dict(cu=_offsets(torch.full((R,), new)), lens=lens.to(torch.int32).to(DEV), table=table.to(DEV), T=R * new,
                  q=_normal(g, R * new, H, d), cache=_fill_cache(g, pages, Hk, page, d), bits=_tree_bits(R, new, seed) if case["tree"] else None)
    return s


def run(s):
    return (_own if own else _plain)(s)


def _own(s):
    import paper_2409_15097_amd as bbm
    op = s["op"]
    if op == "slots":
        r = bbm.bbm_build_slots(s["ctx_lens"], s["new_lens"], s["table"], s["free"], s["free_at"], s["T"], s["page"])
        return {"table": s["table"], "cu": r.cu_new, "lens": r.lens, "positions": r.positions, "slots": r.slots, "free_next": r.free_next}
    if op == "rope":
        q, k = bbm.bbm_rope(s["q"], s["k"], s["positions"], s["freqs"], interleaved=s["pairs"] == "even", mscale=s["mscale"], inverse=s["inverse"])
        return {"q": q, "k": k}
    if op in ("prompt", "train"):
        o, lse = bbm.bbm_prompt_attn_fwd(s["q"], s["k"], s["v"], s["cu"])
        if op == "prompt":
            return {"o": o, "lse": lse}
        dq, dk, dv = bbm.bbm_prompt_attn_bwd(s["q"], s["k"], s["v"], o, s["d_o"], lse, s["cu"])
        return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    cache = bbm.KV4Cache(**s["cache"])
    if op == "append":
        bbm.bbm_kv4_append(s["k"], s["v"], s["slots"], cache)
        k, v = bbm.bbm_kv4_read(s["slots"], cache)
        return {"k": k, "v": v}
    o, lse = bbm.bbm_kv4_attn(s["q"], cache, s["table"], s["lens"], s["cu"], mask=s["bits"], max_len=s["L"])
    return {"o": o, "lse": lse}


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end (angles in 64)


def _plain(s):
    return {"slots": _plain_slots, "rope": _plain_rope, "prompt": _plain_prompt, "train": _plain_prompt, "append": _plain_append, "cached": _plain_cached}[s["op"]](s)


def _plain_slots(s):
    ctx, new, page, table = s["ctx_lens"].long(), s["new_lens"].long(), s["page"], s["table"]
    R, width = table.shape
    lens, ends = ctx + new, new.cumsum(0)
    held, want = (-(-ctx // page)).clamp(max=width), (-(-lens // page)).clamp(max=width)
    taken = want - held
    first = s["free_at"].long() + taken.cumsum(0) - taken
    col = torch.arange(width, device=DEV)
    at = first[:, None] + col - held[:, None]
    fresh = (col >= held[:, None]) & (col < want[:, None])
    n_free = s["free"].numel()
    table = torch.where(fresh, torch.where(at < n_free, s["free"][at.clamp(0, n_free - 1)], -1), table)
    t = torch.arange(s["T"], device=DEV)
    r = torch.searchsorted(ends, t, right=True)
    real, r = r < R, r.clamp(max=R - 1)
    pos = torch.where(real, ctx[r] + t - (ends - new)[r], 0)
    entry = table[r, (pos // page).clamp(max=width - 1)].long()
    slots = torch.where(real & (entry >= 0) & (pos // page < width), entry * page + pos % page, -1)
    cu = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), ends])
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    return {"table": table, "cu": i32(cu), "lens": i32(lens), "positions": i32(pos), "slots": i32(slots), "free_next": i32(s["free_at"] + taken.sum())}


def _plain_rope(s):
    angle = s["positions"].double()[:, None] * s["freqs"].double()
    cos, sin = (angle.cos() * s["mscale"]).float()[:, None], (angle.sin() * s["mscale"]).float()[:, None]
    if s["inverse"]:
        sin = -sin

    def turn(x):
        rot = s["rot"]
        x = x.float()
        y = x.clone()
        a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if s["pairs"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., b] * cos + x[..., a] * sin
        return y.to(torch.bfloat16)
    return {"q": turn(s["q"]), "k": turn(s["k"])}


def _padded(cu, L, T):
    """[R, L]: the packed row of each request's tokens, T where a request is shorter."""
    i = torch.arange(L, device=DEV)
    begin, end = cu[:-1, None].long(), cu[1:, None].long()
    return torch.where(begin + i < end, begin + i, T)


def _take(x, rows, groups):
    """Packed [T, H, d] as [R, groups, H / groups * L, d] in 32 bits, zeros behind each request's end."""
    R, L = rows.shape
    H, d = x.shape[1:]
    x = torch.cat([x.float(), torch.zeros(1, H, d, device=DEV)])[rows]
    return x.permute(0, 2, 1, 3).reshape(R, groups, H // groups * L, d)


def _put(x, rows, T, H):
    """The way back."""
    R, L = rows.shape
    x = x.reshape(R, H, L, -1).permute(0, 2, 1, 3)
    out = torch.empty(T + 1, H, x.shape[-1], device=DEV)
    out[rows] = x
    return out[:T]


def _plain_prompt(s):
    H, Hk, d, L, T = s["H"], s["Hk"], s["d"], s["L"], s["T"]
    rows, scale, G = _padded(s["cu"], s["L"], s["T"]), s["d"] ** -0.5, s["H"] // s["Hk"]
    R = rows.shape[0]
    q, k, v = (_take(s[x], rows, Hk) for x in "qkv")
    i = torch.arange(L, device=DEV)
    hidden = (i > i[:, None]).repeat(G, 1)
    x = (q @ k.transpose(-1, -2).contiguous()).mul_(scale).masked_fill_(hidden, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = top + total.log()
    p = p.div_(total)
    o = p @ v
    out = {"o": _put(o, rows, T, H).to(torch.bfloat16), "lse": _put(lse, rows, T, H)[..., 0].t().contiguous()}
    if s["op"] == "train":
        d_o = _take(s["d_o"], rows, Hk)
        dv = p.transpose(-1, -2).contiguous() @ d_o
        ds = d_o @ v.transpose(-1, -2).contiguous()
        ds = ds.sub_((d_o * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
        out |= {"dq": _put(ds @ k, rows, T, H).to(torch.bfloat16), "dk": _put(ds.transpose(-1, -2).contiguous() @ q, rows, T, Hk).to(torch.bfloat16),
                "dv": _put(dv, rows, T, Hk).to(torch.bfloat16)}
    return out


def _plain_append(s):
    def held(x):
        T, Hk, d = x.shape
        x = x.float().view(T, Hk, d // 32, 32)
        m, e = torch.frexp(x.abs().amax(-1, keepdim=True))              # amax = m 2^e, m in [0.5, 1)
        e = (torch.where(m > 0.875, e - 2, e - 3)).clamp(-120, 125)
        scale = ((e + 127) << 23).to(torch.int32).view(torch.float32)
        y = x.abs() / scale
        step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
        y = ((y / step).round() * step).clamp(max=6)                      # round() takes ties to even
        y = torch.copysign(y * scale, x).to(torch.bfloat16).view(T, Hk, d)
        return torch.where((s["slots"] >= 0)[:, None, None], y, torch.zeros_like(y))
    return {"k": held(s["k"]), "v": held(s["v"])}


def _values(codes, exps):
    """Values of codes [..., d/2] with scale bytes [..., d/32], in 32 bits."""
    lut = torch.tensor(GRID + tuple(-x for x in GRID), device=DEV)
    x = lut[torch.stack([codes & 15, codes >> 4], -1).int()].flatten(-2)
    return (x.unflatten(-1, (-1, 32)) * (exps.int() << 23).view(torch.float32)[..., None]).flatten(-2)


def _plain_cached(s):
    H, Hk, d, new, T, table, c = s["H"], s["Hk"], s["d"], s["new"], s["T"], s["table"].long(), s["cache"]
    rows, G, R = _padded(s["cu"], s["new"], s["T"]), s["H"] // s["Hk"], table.shape[0]
    keys = table.shape[1] * s["page"]
    k = _values(c["k"][table], c["k_scale"][table]).transpose(1, 2).reshape(R, Hk, keys, d)
    v = _values(c["v"][table], c["v_scale"].transpose(-1, -2)[table]).transpose(1, 2).reshape(R, Hk, keys, d)
    q = _take(s["q"], rows, Hk)
    j = torch.arange(keys, device=DEV)[None, None]
    prefix, i = (s["lens"] - new).long()[:, None, None], torch.arange(new, device=DEV)[None, :, None]
    if s["bits"] is None:
        seen = j <= prefix + i
    else:
        own_j = (j - prefix).clamp(0, new - 1).expand(R, new, keys)
        word = s["bits"].view(R, new, -1).gather(2, own_j // 64)
        seen = (j < prefix) | ((word >> (own_j % 64) & 1 != 0) & (j < prefix + new))
    x = (q @ k.transpose(-1, -2).contiguous()).mul_(d ** -0.5).view(R, Hk, G, new, keys).masked_fill_(~seen[:, None, None], -math.inf).view(R, Hk, G * new, keys)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o, lse = (p @ v) / total, top + total.log()
    return {"o": _put(o, rows, T, H).to(torch.bfloat16), "lse": _put(lse, rows, T, H)[..., 0].t().contiguous()}


def work(case):
    op = case["op"]
    if op == "slots":
        R, T = case["R"], int(_step_lengths(case).sum())
        pages = T / case["page"]                                         # an entry from the free list and one to the table for each
        return {"bytes": 4 * (2 * R + 2 * R + 1 + 2 * T + R + 2 * pages), "flops": 0}
    if op == "rope":
        n = case["T"] * (case["H"] + case["Hk"])
        return {"bytes": 4 * n * case["d"] + 4 * case["T"], "flops": 3 * n * case["rot"]}
    if op in ("prompt", "train"):
        n = _lengths(case)
        T, pairs = int(n.sum()), int((n * (n + 1) // 2).sum())
        H, Hk, d = case["H"], case["Hk"], case["d"]
        rows = 2 * d * T * (2 * H + 2 * Hk) + 4 * T * H                  # q, o, k, v; lse
        if op == "train":
            rows += 2 * d * T * (2 * H + 2 * Hk)                          # d_o, dq, dk, dv
        return {"bytes": rows, "flops": (14 if op == "train" else 4) * d * H * pairs}
    if op == "append":
        n = 2 * case["T"] * case["Hk"] * case["d"]                        # values in, and values out again; written and read in 4 bits
        return {"bytes": n * (2 + 2 + 2 * 17 / 32) + 8 * case["T"], "flops": 6 * n}
    R, new, H, Hk, d = (case[x] for x in ("R", "new", "H", "Hk", "d"))
    keys = case["L"] + (R - 1) * max(0.75 * case["L"], new)
    return {"bytes": keys * Hk * d * 2 * 17 / 32 + 4 * R * new * H * (d + 1), "flops": 4 * d * H * new * keys}


# ---- the definitions in 64 bits, one request and head group at a time


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op == "rope":
        return {"q": _exact_rope(s, s["q"]), "k": _exact_rope(s, s["k"])}
    if op in ("prompt", "train"):
        return _exact_prompt(s)
    if op == "cached":
        return _exact_cached(s)
    if op == "append":
        return {"k": _exact_append(s, s["k"]), "v": _exact_append(s, s["v"])}
    return None  # whole numbers


def _exact_rope(s, x):
    rot, sign = s["rot"], -1.0 if s["inverse"] else 1.0
    turn = torch.polar(torch.full_like(s["freqs"], s["mscale"], dtype=torch.float64).expand(x.shape[0], -1).contiguous(),
                       sign * torch.outer(s["positions"].double(), s["freqs"].double()))
    head = x[..., :rot].double()
    if s["pairs"] == "half":
        z = torch.complex(head[..., :rot // 2].contiguous(), head[..., rot // 2:].contiguous()) * turn[:, None]
        y = torch.cat([z.real, z.imag], -1)
    else:
        z = torch.complex(head[..., 0::2].contiguous(), head[..., 1::2].contiguous()) * turn[:, None]
        y = torch.stack([z.real, z.imag], -1).flatten(-2)
    return torch.cat([y, x[..., rot:].double()], -1)


def _exact_append(s, x):
    T, Hk, d = x.shape
    x = torch.where((s["slots"] < 0)[:, None, None], 0.0, x.double()).reshape(-1, 32)
    powers = torch.pow(2.0, torch.arange(-120, 126, dtype=torch.float64, device=DEV))
    scale = powers[torch.searchsorted(7 * powers, x.abs().amax(-1)).clamp(max=len(powers) - 1)][:, None]
    grid = torch.tensor(GRID, dtype=torch.float64, device=DEV)
    # a value halfway between codes c and c + 1 goes to the even one of them
    past, at = (grid[1:] + grid[:-1]) / 2, x.abs() / scale
    code = torch.where(torch.arange(7, device=DEV) % 2 == 1, at[..., None] >= past, at[..., None] > past).sum(-1)
    return (grid[code] * scale * x.sign()).view(T, Hk, d)


def _exact_prompt(s):
    G, scale, cu = s["H"] // s["Hk"], 1 / math.sqrt(s["d"]), s["cu"].tolist()
    names = ["o", "dq", "dk", "dv"] if s["op"] == "train" else ["o"]
    out = {n: torch.zeros(s["T"], s["Hk"] if n in ("dk", "dv") else s["H"], s["d"], dtype=torch.float64, device=DEV) for n in names}
    out["lse"] = torch.zeros(s["H"], s["T"], dtype=torch.float64, device=DEV)
    for a, b in zip(cu, cu[1:]):
        unseen = torch.ones(b - a, b - a, dtype=torch.bool, device=DEV).triu(1)
        for h in range(s["H"]):
            q, k, v = s["q"][a:b, h].double(), s["k"][a:b, h // G].double(), s["v"][a:b, h // G].double()
            x = torch.where(unseen, -math.inf, torch.mm(q, k.t()) * scale)
            lse = torch.logsumexp(x, -1)
            p = torch.exp(x - lse[:, None])
            del x
            out["lse"][h, a:b], out["o"][a:b, h] = lse, torch.mm(p, v)
            if s["op"] == "train":
                d_o = s["d_o"][a:b, h].double()
                out["dv"][a:b, h // G] += torch.mm(p.t(), d_o)
                ds = p * (torch.mm(d_o, v.t()) - (d_o * out["o"][a:b, h]).sum(-1)[:, None]) * scale
                out["dq"][a:b, h] = torch.mm(ds, k)
                out["dk"][a:b, h // G] += torch.mm(ds.t(), q)
    return out


def _exact_cached(s):
    if s["R"] * s["Hk"] > 4096:
        return None
    H, Hk, d, new, c = s["H"], s["Hk"], s["d"], s["new"], s["cache"]
    grid = torch.tensor(GRID, dtype=torch.float64, device=DEV)
    o = torch.zeros(s["T"], H, d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(H, s["T"], dtype=torch.float64, device=DEV)

    def decode(codes, exps):                                               # [n, Hk, page, d/2], [n, Hk, page, d/32] -> [Hk, n * page, d]
        nibbles = torch.zeros(*codes.shape[:-1], d, dtype=torch.int64, device=DEV)
        nibbles[..., 0::2], nibbles[..., 1::2] = (codes % 16).long(), torch.div(codes, 16, rounding_mode="floor").long()
        x = grid[nibbles % 8] * torch.where(nibbles >= 8, -1.0, 1.0)
        x = x * torch.pow(2.0, exps.double() - 127).repeat_interleave(32, -1)
        return x.movedim(1, 0).flatten(1, 2)
    for r, n in enumerate(s["lens"].tolist()):
        ids = s["table"][r, :-(-n // s["page"])].long()
        k = decode(c["k"][ids], c["k_scale"][ids])[:, :n]
        v = decode(c["v"][ids], c["v_scale"][ids].transpose(-1, -2))[:, :n]
        seen = torch.ones(new, n, dtype=torch.bool, device=DEV)
        if s["bits"] is None:
            seen[:, n - new:] = torch.ones(new, new, dtype=torch.bool, device=DEV).tril()
        else:
            at = torch.arange(new, device=DEV)
            seen[:, n - new:] = (s["bits"][r * new:(r + 1) * new][:, at // 64] >> (at % 64)) % 2 != 0
        q = s["q"][r * new:(r + 1) * new].double().transpose(0, 1).reshape(Hk, -1, d)     # [Hk, G * new, d]
        x = torch.bmm(q, k.transpose(1, 2).contiguous()).view(H, new, n) / math.sqrt(d)
        x = torch.where(seen, x, -math.inf)
        z = torch.logsumexp(x, -1)
        w = torch.exp(x - z[..., None]).view(Hk, -1, n)
        o[r * new:(r + 1) * new] = torch.bmm(w, v.contiguous()).view(H, new, d).transpose(0, 1)
        lse[:, r * new:(r + 1) * new] = z
    return {"o": o, "lse": lse}
