"""Operators of serving over the 4-bit cache, as cases to time, with their plain forms and their values in 64 bits.

Requests lie in a paged cache of keys and values in 4 bits (groups of 32 values: a scale byte s = e + 127, codes of x / 2^e on 0, .5, 1, 1.5, 2, 3, 4, 6,
the sign in bit 3, element 2i in the low half of byte i).  A case names an operator and its sizes:

* ``shared``   attention of new tokens where groups of requests have the same pages for a long prefix;
* ``weights``  the attention weight that each key of the cache gets from the new tokens, added to what it had;
* ``evict``    of requests that are longer than a budget the keys of least accumulated weight go, the rest moves together, pages go back.

Head sizes 64 and 128, bf16 and the softmax scale 1/sqrt(d) are those of the rest of the library; queries are N(0,1).
"""
import math

import torch

own = False

DEV = "cuda"
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    case = lambda name, op, **more: dict(name=name, op=op, **more)  # noqa: E731
    return [
        # four answers of one short prompt: the smallest call, all launches and latency
        case("shared-answers", "shared", S=1, R=4, lone=0, prefix=512, own=48, new=1, H=32, Hk=8, d=128, page=16),
        # a server whose requests begin with the same instructions, a few of them with none
        case("shared-system", "shared", S=1, R=67, lone=3, prefix=8192, own=1000, new=1, H=32, Hk=8, d=128, page=64),
        # several documents, each with its own questions, in smaller heads
        case("shared-groups", "shared", S=7, R=61, lone=0, prefix=4096, own=333, new=1, H=16, Hk=4, d=64, page=32),
        # drafts of up to 9 tokens to be verified, for many answers of one document
        case("shared-drafts", "shared", S=2, R=32, lone=0, prefix=6000, own=500, new=9, H=32, Hk=8, d=128, page=16),
        # a long document for as many requests as a step holds: the largest
        case("shared-long", "shared", S=1, R=256, lone=0, prefix=32768, own=500, new=1, H=32, Hk=8, d=128, page=128),
        # one long answer alone
        case("weights-one", "weights", S=0, R=1, lone=1, prefix=0, own=2000, new=1, H=16, Hk=4, d=64, page=16),
        # a decoding step of a server
        case("weights-decode", "weights", S=0, R=64, lone=64, prefix=0, own=8192, new=1, H=32, Hk=8, d=128, page=64),
        # a decoding step behind a shared prefix
        case("weights-shared", "weights", S=1, R=67, lone=3, prefix=8192, own=1000, new=1, H=32, Hk=8, d=128, page=64),
        # a part of a prompt behind what the cache holds already
        case("weights-prompt", "weights", S=0, R=3, lone=3, prefix=0, own=6000, new=1500, H=32, Hk=8, d=128, page=32),
        # one answer has reached its budget
        case("evict-one", "evict", R=1, n=1040, budget=1024, recent=128, first=4, Hk=4, d=64, page=16),
        # the requests of a server, a page over their budget or not yet
        case("evict-step", "evict", R=64, n=2112, budget=2048, recent=256, first=4, Hk=8, d=128, page=64),
        # long prompts are thinned to an eighth
        case("evict-prompts", "evict", R=16, n=32000, budget=4000, recent=500, first=64, Hk=8, d=128, page=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["shared", "shared", "weights", "evict"])
    d = rng.choice([64, 128])
    Hk = rng.choice([1, 2, 4, 8])
    H = Hk * rng.choice([1, 2, 3, 4, 8])
    page = rng.choice([16, 32, 64, 128])
    if op == "evict":
        budget = _log(rng, 16, 8192)
        n = min(budget + (_log(rng, 1, 128) if rng.random() < 0.5 else _log(rng, 1, 8 * budget)), 32000)
        case = dict(op=op, R=_log(rng, 1, 64), n=n, budget=budget, recent=rng.randint(0, budget // 2), first=rng.choice([0, 4, 64]), Hk=Hk, d=d, page=page)
    elif op == "weights" and rng.random() < 0.5:
        new, R = rng.choice([1, 1, 2, _log(rng, 1, 1500)]), _log(rng, 1, 128)
        case = dict(op=op, S=0, R=R, lone=R, prefix=0, own=max(new, _log(rng, 1, 16384)), new=new, H=H, Hk=Hk, d=d, page=page)
    else:
        new, R = rng.choice([1, 1, 1, 2, _log(rng, 1, 16)]), _log(rng, 1, 256)
        S = rng.randint(1, min(R, 8))
        case = dict(op=op, S=S, R=R, lone=rng.randint(0, min(3, R - S)), prefix=_log(rng, 16, 32768), own=max(new, _log(rng, 1, 1000)), new=new, H=H, Hk=Hk, d=d, page=page)
    # (fewer requests where it would be more than the listed ones are)
    listed_work = [work(c) for c in listed() if c["op"] == op]
    while case["R"] > 1 and any(work(case)[x] > max(w[x] for w in listed_work) for x in ("bytes", "flops")):
        case["R"] //= 2
        if op != "evict":
            case["S"] = min(case["S"], case["R"])
            case["lone"] = min(case["lone"], case["R"] - case["S"]) if case["S"] else case["R"]
    return case


def _sizes(case):
    """Of a case, the same for every seed: requests of each group, keys they share (whole pages), new tokens and own keys of each request."""
    S, R, lone = case["S"], case["R"], case["lone"]
    members = R - lone
    cuts = torch.tensor([0] + [s + (members - S) * s * (s + 1) // (S * (S + 1)) for s in range(1, S + 1)]) if S else torch.zeros(1, dtype=torch.int64)
    s = torch.arange(S, dtype=torch.float64)
    shared = ((case["prefix"] * (1 - 0.4 * s / max(1, S))).to(torch.int64) // case["page"]) * case["page"]
    r = torch.arange(R)
    new = torch.ones(R, dtype=torch.int64) if case["new"] == 1 else 1 + r * 7919 % case["new"]
    if case["new"] > 1:
        new[0] = case["new"]
    own_keys = (case["own"] * (0.5 + 0.5 * ((r * 7 + 1) % (R + 1)).double() / (R + 1))).round().to(torch.int64)
    own_keys[0] = case["own"]
    return cuts, shared, new, torch.maximum(own_keys, new)


def _evict_lens(case):
    r = torch.arange(case["R"], dtype=torch.float64)
    lens = (case["n"] * (1 - 0.25 * ((r * 7) % case["R"]) / case["R"])).round().to(torch.int64)
    return lens.clamp(1, case["n"])


def _offsets(n):
    return torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(torch.int32)


def _cache(g, pages, Hk, page, d):
    """Pages as a program finds them: codes and scales of N(0,1) data, in the layout of the cache."""
    codes = lambda: torch.randint(0, 256, (pages, Hk, page, d // 2), generator=g, device=DEV, dtype=torch.uint8)  # noqa: E731
    exps = lambda *s: torch.randint(124, 127, s, generator=g, device=DEV, dtype=torch.uint8)  # noqa: E731
    return {"k": codes(), "k_scale": exps(pages, Hk, page, d // 32), "v": codes(), "v_scale": exps(pages, Hk, d // 32, page)}


def prepare(case, seed):
    h = torch.Generator().manual_seed(seed * 7919 + 21)
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 22)
    Hk, d, page, R = case["Hk"], case["d"], case["page"], case["R"]
    s = dict(case, seed=seed)
    dev = lambda x: x.to(torch.int32).to(DEV)  # noqa: E731
    if case["op"] == "evict":
        lens = _evict_lens(case)[torch.randperm(R, generator=h)]
        width = -(-case["n"] // page)
        pages = R * width + 2
        ids = torch.randperm(pages, generator=h)
        # (weights as they add up: few keys with much, many with little)
        weights = torch.rand(pages, Hk, page, generator=g, device=DEV).pow_(8).mul_(50)
        free = torch.cat([ids[:R * width], ids])                             # those taken lie in front of free_at
        return s | dict(lens=dev(lens), table=dev(ids[:R * width].view(R, width)), cache=_cache(g, pages, Hk, page, d), weights=weights, keep_first=dev(torch.full((R,), case["first"])),
                        free=dev(free), free_at=dev(torch.tensor([R * width])))
    cuts, shared, new, own_keys = _sizes(case)
    S, H = case["S"], case["H"]
    group = torch.bucketize(torch.arange(R), cuts, right=True) - 1
    in_front = torch.where(group < S, torch.cat([shared, torch.zeros(1, dtype=torch.int64)])[group.clamp(max=S)], 0)
    lens = in_front + own_keys
    width = int((-(-lens // page)).max())
    col, held = torch.arange(width), in_front // page
    prefix_pages = int((shared // page).sum())
    own_pages = -(-own_keys // page)
    pages = prefix_pages + int(own_pages.sum()) + 3
    ids = torch.randperm(pages, generator=h)
    prefix_at, own_at = torch.cat([torch.zeros(1, dtype=torch.int64), (shared // page).cumsum(0)]), prefix_pages + own_pages.cumsum(0) - own_pages
    at = torch.where(col < held[:, None], prefix_at[group.clamp(max=S)][:, None] + col, own_at[:, None] + col - held[:, None])
    table = torch.where(col < (held + own_pages)[:, None], ids[at.clamp(max=pages - 1)], -1)
    T = int(new.sum())
    s |= dict(T=T, cu=_offsets(new).to(DEV), lens=dev(lens), table=dev(table), group_cu=dev(cuts), shared=dev(shared), group=group.to(DEV), cache=_cache(g, pages, Hk, page, d),
              members=max([int(x) for x in cuts.diff()], default=0), q=torch.randn(T, H, d, generator=g, device=DEV).to(torch.bfloat16))
    if case["op"] == "weights":
        s["lse"] = _plain_attention(s)["lse"]                                # what the attention of the same step gave
        s["weights"] = torch.rand(pages, Hk, page, generator=g, device=DEV)
        s["sums"] = s["weights"].clone()
    return s


def run(s):
    return (_own if own else _plain)(s)


def _own(s):
    import paper_2409_15097_amd as bbm
    cache = bbm.KV4Cache(**s["cache"])
    if s["op"] == "shared":
        o, lse = bbm.bbm_kv4_shared_attn(s["q"], cache, s["table"], s["lens"], s["cu"], s["group_cu"], s["shared"], max_shared=s["prefix"], max_own=s["own"])
        return {"o": o, "lse": lse}
    if s["op"] == "weights":
        groups = dict(group_cu=s["group_cu"], shared_lens=s["shared"], max_shared=s["prefix"]) if s["S"] else {}
        return {"weights": bbm.bbm_kv4_weights(s["q"], s["lse"], cache, s["table"], s["lens"], s["cu"], s["weights"], out=s["sums"], decay=0.875, max_own=s["own"], **groups)}
    r = bbm.bbm_kv4_evict(cache, s["weights"], s["table"], s["lens"], s["budget"], recent=s["recent"], first=s["keep_first"], free_pages=s["free"], free_at=s["free_at"],
                          max_len=s["n"])
    return {**s["cache"], "weights": s["weights"], "lens": r.lens, "free": s["free"], "free_next": r.free_next}


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end


def _plain(s):
    return {"shared": _plain_shared, "weights": _plain_weights, "evict": _plain_evict}[s["op"]](s)


def _values(codes, exps):
    """Values of codes [..., d/2] with scale bytes [..., d/32], in 32 bits."""
    lut = torch.tensor(GRID + tuple(-x for x in GRID), device=DEV)
    x = lut[torch.stack([codes & 15, codes >> 4], -1).int()].flatten(-2)
    return (x.unflatten(-1, (-1, 32)) * (exps.int() << 23).view(torch.float32)[..., None]).flatten(-2)


def _keys(s, pages):
    """Of pages [n, m] of the cache: keys [n, Hk, m * page, d]."""
    return _values(s["cache"]["k"][pages], s["cache"]["k_scale"][pages]).transpose(1, 2).flatten(2, 3)


def _vals(s, pages):
    return _values(s["cache"]["v"][pages], s["cache"]["v_scale"].transpose(-1, -2)[pages]).transpose(1, 2).flatten(2, 3)


def _rows(begin, end, most, T):
    """[n, most]: rows begin .. end - 1 of each, T behind them."""
    i = torch.arange(most, device=DEV)
    return torch.where(begin[:, None] + i < end[:, None], begin[:, None] + i, T)


def _queries(s, rows):
    """[n, Hk, G * m, d] of rows [n, m], zeros where there is none."""
    n, m = rows.shape
    x = torch.cat([s["q"].float(), torch.zeros(1, s["H"], s["d"], device=DEV)])[rows]
    return x.permute(0, 2, 1, 3).reshape(n, s["Hk"], s["H"] // s["Hk"] * m, s["d"])


def _packed(s, x, rows):
    """[n, Hk, G * m, e] back to [T + 1, H, e]; the last row takes what belongs to nobody."""
    n, m = rows.shape
    x = x.reshape(n, s["H"], m, -1).permute(0, 2, 1, 3)
    out = x.new_zeros(s["T"] + 1, s["H"], x.shape[-1])
    out[rows] = x
    return out


def _scores(s):
    """Scores over the shared keys of each group and over the own keys of each request, -infinity where a query does not see one: (scores, rows, pages) of both."""
    page, T, cu, table, lens = s["page"], s["T"], s["cu"].long(), s["table"].long(), s["lens"].long()
    shared = torch.cat([s["shared"].long(), torch.zeros(1, dtype=torch.int64, device=DEV)])
    front = torch.where(s["group"] < s["S"], shared[s["group"].clamp(max=s["S"])], 0)
    rows = _rows(cu[:-1], cu[1:], s["new"], T)
    new, width = cu.diff(), -(-s["own"] // page)
    at = (front // page)[:, None] + torch.arange(width, device=DEV)
    pages = table.gather(1, at.clamp(max=table.shape[1] - 1)).clamp(min=0)
    j, i = torch.arange(width * page, device=DEV), torch.arange(s["new"], device=DEV)
    seen = front[:, None, None] + j <= (lens - new)[:, None, None] + i[:, None]
    seen = seen & (i < new[:, None])[:, :, None]
    G = s["H"] // s["Hk"]
    x = (_queries(s, rows) @ _keys(s, pages).transpose(-1, -2).contiguous()).mul_(s["d"] ** -0.5)
    x.masked_fill_(~seen[:, None].repeat(1, 1, G, 1), -math.inf)
    if not s["S"] or s["prefix"] < page:
        return None, (x, rows, pages)
    gc = s["group_cu"].long()
    rows_p = _rows(cu[gc[:-1]], cu[gc[1:]], s["members"] * s["new"], T)
    pages_p = table[gc[:-1], :s["prefix"] // page].clamp(min=0)
    j = torch.arange(pages_p.shape[1] * page, device=DEV)
    y = (_queries(s, rows_p) @ _keys(s, pages_p).transpose(-1, -2).contiguous()).mul_(s["d"] ** -0.5)
    y.masked_fill_((j >= s["shared"].long()[:, None])[:, None, None], -math.inf)
    return (y, rows_p, pages_p), (x, rows, pages)


def _sums(s, part, with_values):
    """(maximum, sum of exponentials, their sum over values) of each row of the packed tensors, over a part of the keys."""
    x, rows, pages = part
    top = x.amax(-1, keepdim=True)
    p = x.sub_(top.clamp(min=-1e30)).exp_()
    total = p.sum(-1, keepdim=True)
    put = lambda y: _packed(s, y, rows)[:s["T"]]  # noqa: E731
    return put(top.clamp(min=-1e30)), put(total), put(p @ _vals(s, pages)) if with_values else None


def _plain_attention(s, with_values=False):
    shared, mine = _scores(s)
    m, l, a = _sums(s, mine, with_values)
    if shared is not None:
        m2, l2, a2 = _sums(s, shared, with_values)
        top = torch.maximum(m, m2)
        f, f2 = torch.where(l > 0, (m - top).exp(), 0.0), torch.where(l2 > 0, (m2 - top).exp(), 0.0)
        m, l = top, l * f + l2 * f2
        a = a * f + a2 * f2 if with_values else None
    out = {"lse": (m + l.log())[..., 0].t().contiguous()}
    if with_values:
        out["o"] = (a / l).to(torch.bfloat16)
    return out


def _plain_shared(s):
    r = _plain_attention(s, True)
    return {"o": r["o"], "lse": r["lse"]}


def _plain_weights(s):
    shared, mine = _scores(s)
    page, Hk, out = s["page"], s["Hk"], s["sums"]
    lse = torch.cat([s["lse"].t(), torch.zeros(1, s["H"], device=DEV)])

    def gained(part):                                                        # [n, Hk, keys]
        x, rows, pages = part
        n, m = rows.shape
        z = lse[rows].permute(0, 2, 1).reshape(n, Hk, -1, 1)
        p = x.sub_(z).exp_().view(n, Hk, -1, m, x.shape[-1])
        return p.mul_((rows < s["T"])[:, None, None, :, None]).sum((2, 3))

    lens, new = s["lens"].long(), s["cu"].long().diff()

    def add(part, begin, end, fresh):
        """To the weights of keys begin .. end - 1 of each row of pages; those from `fresh` on had none."""
        w, pages = gained(part), part[2]
        n, m = pages.shape
        j = torch.arange(m * page, device=DEV) + begin[:, None]
        old = s["weights"][pages].transpose(1, 2).reshape(n, Hk, m * page)
        old = torch.where((j < fresh[:, None])[:, None], old * 0.875, 0.0)
        there = (j < end[:, None])[:, None, :, None].expand(n, Hk, m * page, 1).reshape(n, Hk, m, page).transpose(1, 2)
        # (what lies behind a request's end keeps its value; a page that is nobody's is written with what it holds)
        new_w = torch.where(there, (old + w).view(n, Hk, m, page).transpose(1, 2), out[pages])
        taken = (begin[:, None] + torch.arange(m, device=DEV) * page) < end[:, None]
        spare = torch.where(taken, pages, out.shape[0])
        grown = torch.cat([out, out.new_zeros(1, Hk, page)])
        grown[spare] = new_w
        out.copy_(grown[:-1])

    sh = torch.cat([s["shared"].long(), torch.zeros(1, dtype=torch.int64, device=DEV)])
    front = torch.where(s["group"] < s["S"], sh[s["group"].clamp(max=s["S"])], 0)
    add(mine, front, lens, lens - new)
    if shared is not None:
        zero = torch.zeros_like(sh[:-1])
        add(shared, zero, sh[:-1], sh[:-1])
    return {"weights": out}


def _plain_evict(s):
    page, budget, Hk, c = s["page"], s["budget"], s["Hk"], s["cache"]
    lens, first, table = s["lens"].long(), s["keep_first"].long(), s["table"].long()
    R, width = table.shape
    N = width * page
    b = torch.clamp(first + s["recent"], min=budget)
    active = lens > b
    j = torch.arange(N, device=DEV)
    col = lambda x: x[:, None, None]  # noqa: E731
    w = s["weights"][table].transpose(1, 2).reshape(R, Hk, N)
    mid = (j >= col(first)) & (j < col(lens - s["recent"]))
    order = torch.sort(torch.where(mid, w, -math.inf), dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, j.expand_as(order))
    kept = mid & (rank < col(b - first - s["recent"]))
    edge = col(b - s["recent"])
    holes, movers = mid & ~kept & (j < edge), kept & (j >= edge)
    # the place of the i-th hole, and who moves there
    hole_at = torch.zeros(R, Hk, N + 1, dtype=torch.int64, device=DEV)
    hole_at.scatter_(-1, torch.where(holes, holes.cumsum(-1) - 1, N), j.expand(R, Hk, N))
    to = torch.where(movers, hole_at.gather(-1, (movers.cumsum(-1) - 1).clamp(min=0)), N)
    late = (j >= col(lens - s["recent"])) & (j < col(lens))
    to = torch.where(late, j - col(lens - b), to)
    to = torch.where(col(active), to, N)
    source = torch.cat([j, j.new_zeros(1)]).expand(R, Hk, N + 1).clone().scatter_(-1, to, j.expand(R, Hk, N))[..., :N]
    moved = col(active) & (source != j)

    def take(x):                                                             # [pages, Hk, page, e], in place
        y = x[table].transpose(1, 2).reshape(R, Hk, N, -1)
        y = torch.where(moved[..., None], y.gather(2, source[..., None].expand(R, Hk, N, y.shape[-1])), y)
        x[table] = y.view(R, Hk, width, page, -1).transpose(1, 2)

    take(c["k"]), take(c["v"]), take(c["k_scale"]), take(c["v_scale"].transpose(-1, -2)), take(s["weights"][..., None])
    # pages behind what is kept go back in front of free_at, in the order of requests and positions
    left = torch.where(active, b, lens)
    had, has = -(-lens // page), -(-left // page)
    at = torch.arange(width, device=DEV)
    gone = (at >= has[:, None]) & (at < had[:, None])
    total = gone.sum()
    free_next = s["free_at"].long() - total
    place = torch.where(gone, free_next + gone.flatten().cumsum(0).view(R, width) - 1, s["free"].numel())
    grown = torch.cat([s["free"], s["free"].new_zeros(1)])
    grown[place] = s["table"]
    s["free"].copy_(grown[:-1])
    return {**c, "weights": s["weights"], "lens": left.to(torch.int32), "free": s["free"], "free_next": free_next.to(torch.int32)}


def work(case):
    Hk, d, op = case["Hk"], case["d"], case["op"]
    a_key = d * 17 / 32                                                      # bytes of a key, or a value, of a head
    if op == "evict":
        lens, kept = _evict_lens(case).double(), max(case["budget"], case["first"] + case["recent"])
        over = lens[lens > kept]
        # of the keys between, a share of chosen ones lies behind the edge, as many as there are holes in front of it; the last ones all move
        between = over - case["first"] - case["recent"]
        chosen = kept - case["first"] - case["recent"]
        moves = (over - kept) * chosen / between.clamp(min=1) + case["recent"]
        return {"bytes": Hk * (4 * float(over.sum()) + 2 * (2 * a_key + 4) * float(moves.sum())) + 8 * case["R"], "flops": 0}
    cuts, shared, new, own_keys = _sizes(case)
    T, H = int(new.sum()), case["H"]
    members = cuts.diff()
    rows = torch.stack([new[a:b].sum() for a, b in zip(cuts[:-1], cuts[1:])]) if case["S"] else torch.zeros(0, dtype=torch.int64)
    keys = int((shared * (members > 0)).sum()) + int(own_keys.sum())
    pairs = int((shared * rows).sum()) + int((new * (own_keys - new) + new * (new + 1) // 2).sum())
    io = 2 * T * H * d + 4 * T * H                                            # q and lse
    if op == "shared":
        return {"bytes": keys * Hk * 2 * a_key + io + 2 * T * H * d, "flops": 4 * d * H * pairs}
    return {"bytes": keys * Hk * (a_key + 8) + io, "flops": 2 * d * H * pairs}


# ---- the definitions in 64 bits, one request at a time


def exact(case, seed):
    if case["op"] == "evict":
        return None                                                          # a choice, and copies
    if case["R"] * case["Hk"] > 4096:
        return None
    s = prepare(case, seed)
    H, Hk, d, page, c = s["H"], s["Hk"], s["d"], s["page"], s["cache"]
    grid = torch.tensor(GRID, dtype=torch.float64, device=DEV)

    def decode(codes, exps):                                                 # [n, Hk, page, d/2], [n, Hk, page, d/32] -> [Hk, n * page, d]
        nibbles = torch.zeros(*codes.shape[:-1], d, dtype=torch.int64, device=DEV)
        nibbles[..., 0::2], nibbles[..., 1::2] = (codes % 16).long(), torch.div(codes, 16, rounding_mode="floor").long()
        x = grid[nibbles % 8] * torch.where(nibbles >= 8, -1.0, 1.0)
        return (x * torch.pow(2.0, exps.double() - 127).repeat_interleave(32, -1)).movedim(1, 0).flatten(1, 2)

    weights = s["op"] == "weights"
    o = torch.zeros(s["T"], H, d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(H, s["T"], dtype=torch.float64, device=DEV)
    sums = torch.zeros(c["k"].shape[0] * page, Hk, dtype=torch.float64, device=DEV)
    touched, fresh = torch.zeros_like(sums, dtype=torch.bool), torch.zeros_like(sums, dtype=torch.bool)
    cu = s["cu"].tolist()
    for r, n in enumerate(s["lens"].tolist()):
        a, b = cu[r], cu[r + 1]
        new = b - a
        ids = s["table"][r, :-(-n // page)].long()
        k = decode(c["k"][ids], c["k_scale"][ids])[:, :n]
        seen = torch.ones(new, n, dtype=torch.bool, device=DEV)
        seen[:, n - new:] = torch.ones(new, new, dtype=torch.bool, device=DEV).tril()
        q = s["q"][a:b].double().transpose(0, 1).reshape(Hk, -1, d)            # [Hk, G * new, d]
        x = torch.bmm(q, k.transpose(1, 2).contiguous()).view(H, new, n) / math.sqrt(d)
        x = torch.where(seen, x, -math.inf)
        if weights:
            p = torch.exp(x - s["lse"][:, a:b, None].double()).view(Hk, -1, n).sum(1)   # [Hk, n]
            slot = (ids[:, None] * page + torch.arange(page, device=DEV)).flatten()[:n]
            sums[slot] += p.t()
            touched[slot], fresh[slot[n - new:]] = True, True
            continue
        z = torch.logsumexp(x, -1)
        v = decode(c["v"][ids], c["v_scale"][ids].transpose(-1, -2))[:, :n].contiguous()
        o[a:b] = torch.bmm(torch.exp(x - z[..., None]).view(Hk, -1, n), v).view(H, new, d).transpose(0, 1)
        lse[:, a:b] = z
    if not weights:
        return {"o": o, "lse": lse}
    old = s["weights"].double().transpose(1, 2).reshape(-1, Hk)
    old = torch.where(fresh, 0.0, torch.where(touched, 0.875 * old, old))
    return {"weights": (old + sums).view(-1, page, Hk).transpose(1, 2).contiguous()}
