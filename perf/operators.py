"""The decode side of the compacted cache, as cases that can be timed: normalised and rotated queries and keys, a token's
rows appended to a paged cache, attention of one new token over it, and eviction by accumulated attention.

``own`` false: plain torch operations in 32 bits. ``own`` true: the library's calls.
"""
import math

import torch

own = False

# (query heads, KV heads, head dim): a small model, 8B-class and 70B-class grouped-query shapes, odd and wide groups
SHAPES = ((8, 2, 64), (32, 8, 128), (64, 8, 128), (28, 4, 128), (24, 2, 128), (12, 4, 64))
EPS = 1e-6
POSITIONS = 1 << 17          # rows of the angle tables
BYTES = 1 << 30              # keys and values of the largest drawn cache


def _case(kind, name=None, Hq=32, Hkv=8, d=128, B=1, L=1, page=16, norm=False, ragged=False, w=32, c=10, budget=1):
    case = dict(kind=kind, Hq=Hq, Hkv=Hkv, d=d, B=B, L=L, page=page, norm=norm, ragged=ragged, w=w, c=c, budget=budget)
    return case if name is None else dict(case, name=name)


def listed():
    return [
        # queries and keys of a prompt's layer before its cache is compressed: an ordinary prompt, seven heads a group
        _case("rotate", "rotate 2k", Hq=28, Hkv=4, L=2048),
        # the same of a 32K document, for a model that normalises each head
        _case("rotate", "rotate 32k", L=32768, norm=True),
        # the smallest call of a decode step: one user of a small model
        _case("append", "append 1", Hq=8, Hkv=2, d=64, L=257, norm=True),
        # a full decode batch of a 70B-class model
        _case("append", "append 64", Hq=64, B=64, L=1025),
        # one user whose 32K prompt was compressed to a tenth, some hundred tokens later
        _case("attend", "attend 1 x 3.5k", L=3501),
        # a batch of 70B-class sequences of different lengths, pages of 64 rows
        _case("attend", "attend 9 ragged 8k", Hq=64, B=9, L=8192, page=64, ragged=True),
        # a full decode batch at a budget of 4096 rows a head
        _case("attend", "attend 64 x 4k", B=64, L=4160),
        # one user whose 128K document was not compressed
        _case("attend", "attend 1 x 128k", L=131007),
        # a batch that keeps the sums that eviction goes by, seven heads a group
        _case("weigh", "weigh 8 x 4k", Hq=28, Hkv=4, B=8, L=4352),
        # a layer of a decode step: the token's rows are appended and attended to, with the sums
        _case("step", "step 16 x 2k", B=16, L=2185, norm=True, ragged=True),
        # back to a tenth of a 32K prompt after 256 tokens, in chunks of 10
        _case("evict", "evict 1 x 3.5k c10", L=3532, budget=3276),
        # a batch back to 4096 rows a head after 256 tokens, row by row
        _case("evict", "evict 32 x 4k c1", B=32, L=4352, c=1, budget=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of these ranges."""
    kind = rng.choice(("rotate", "append", "attend", "attend", "attend", "weigh", "step", "evict", "evict"))
    Hq, Hkv, d = rng.choice(SHAPES)
    case = _case(kind, Hq=Hq, Hkv=Hkv, d=d, page=rng.choice((8, 16, 16, 32, 64, 100)), norm=rng.random() < 0.5)
    if kind == "rotate":
        return dict(case, L=min(_log(rng, 64, 32768), 32768 * 40 // (Hq + Hkv)))
    case.update(B=_log(rng, 1, 64), ragged=rng.random() < 0.5)
    if kind == "append":
        return dict(case, L=_log(rng, 16, 2048))
    case["L"] = _log(rng, 64, min(131072, BYTES // (case["B"] * Hkv * d * 4)))
    if kind in ("weigh", "step", "evict"):
        case["B"] = min(case["B"], 32)
        case["L"] = min(case["L"], 16384)
    if kind == "evict":
        c = rng.choice((1, 1, 5, 8, 10, 16, 20))
        w = rng.choice((4, 16, 32, 64))
        L = max(case["L"], 2 * (w + c))
        case.update(w=w, c=c, L=L, budget=max(w + c, int(L * rng.uniform(0.4, 0.98))))
    return case


def _lengths(case):
    """Rows of each (sequence, head): sequences differ where the batch is ragged, and heads by the clipped chunk that some kept."""
    B, Hkv, L = case["B"], case["Hkv"], case["L"]
    seq = [L if not case["ragged"] or b == 0 else max(1, L - int(0.9 * L * ((b * 0.6180339887) % 1.0))) for b in range(B)]
    return [[max(1, n - (6 if h % 3 == 1 else 0)) for h in range(Hkv)] for n in seq]


def _angles(d, device):
    inv = 500000.0 ** (-torch.arange(0, d, 2, device=device, dtype=torch.float64) / d)
    a = torch.arange(POSITIONS, device=device, dtype=torch.float64)[:, None] * inv
    return a.cos().float(), a.sin().float()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    Hq, Hkv, d, B, L, page, kind = (case[k] for k in ("Hq", "Hkv", "d", "B", "L", "page", "kind"))
    dev, bf16, i32 = "cuda", torch.bfloat16, torch.int32
    s = {"case": case}

    def rand(*shape):
        return torch.randn(*shape, device=dev, generator=g, dtype=torch.float32).to(bf16)

    if kind in ("rotate", "append", "step"):
        n = L if kind == "rotate" else B
        s["qkv"] = torch.randn(n, (Hq + 2 * Hkv) * d, device=dev, generator=g, dtype=bf16)
        s["cos"], s["sin"] = _angles(d, dev)
        first = int(torch.randint(0, POSITIONS - 2 * L, (1,), device=dev, generator=g))
        s["pos"] = torch.arange(first, first + n, device=dev, dtype=i32) if kind == "rotate" else torch.randint(L, POSITIONS, (n,), device=dev, generator=g).to(i32)
        s["gq"] = (1.0 + 0.2 * rand(d).float()).to(bf16) if case["norm"] else None
        s["gk"] = (1.0 + 0.2 * rand(d).float()).to(bf16) if case["norm"] else None
    if kind == "rotate":
        return s
    per = -(-L // page) + 1
    pages = B * per + 3
    s["K"] = torch.randn(pages, page, Hkv, d, device=dev, dtype=bf16, generator=g)
    s["V"] = torch.randn(pages, page, Hkv, d, device=dev, dtype=bf16, generator=g)
    s["table"] = torch.randperm(pages, device=dev, generator=g)[: B * per].view(B, per).to(i32).contiguous()
    s["len"] = torch.tensor(_lengths(case), device=dev, dtype=i32)
    if kind in ("attend", "weigh"):
        # the keys of some rows lie along a direction that their queries share, so that attention is spread unevenly
        u = torch.nn.functional.normalize(torch.randn(Hkv, d, device=dev, generator=g), dim=-1)
        lead = torch.randn(pages, page, Hkv, 1, device=dev, generator=g).mul_(0.5 * math.sqrt(d)).to(bf16)
        s["K"] += lead * u.to(bf16)
        s["q"] = (torch.randn(B, Hkv, Hq // Hkv, d, device=dev, generator=g) + 4.0 * u[:, None]).to(bf16).view(B, Hq, d)
    if kind in ("weigh", "step", "evict"):
        # what earlier steps left: spread over orders of magnitude, nothing for many rows, zero behind the last row
        x = torch.randn(B, Hkv, per * page, device=dev, generator=g).mul_(2.0).sub_(3.0).exp_()
        x[torch.rand(B, Hkv, per * page, device=dev, generator=g) < 0.1] = 0.0
        x[torch.arange(per * page, device=dev) >= s["len"][:, :, None]] = 0.0
        s["weights"] = x
    if kind == "evict":
        s["weights0"], s["len0"] = s["weights"].clone(), s["len"].clone()
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _turn(x, gain, cos, sin):
    """x [n, H, d] in 32 bits, cos and sin [n, d / 2]."""
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()
    a, b = x.chunk(2, -1)
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def _rotate(s):
    Hq, Hkv, d = (s["case"][k] for k in ("Hq", "Hkv", "d"))
    x = s["qkv"].view(-1, Hq + 2 * Hkv, d)
    cos, sin = s["cos"][s["pos"].long()][:, None], s["sin"][s["pos"].long()][:, None]
    q = _turn(x[:, :Hq].float(), s["gq"], cos, sin)
    k = _turn(x[:, Hq:Hq + Hkv].float(), s["gk"], cos, sin)
    return q.bfloat16(), k.bfloat16()


def _rows(s, row):
    """(page, slot) of rows [B, Hkv, n] of their sequences."""
    page = s["case"]["page"]
    table = s["table"][:, None, :].expand(-1, row.shape[1], -1).long()
    return table.gather(2, row // page), row % page


def _append(s):
    Hq, Hkv, d, B = (s["case"][k] for k in ("Hq", "Hkv", "d", "B"))
    q, k = _rotate(s)
    v = s["qkv"].view(B, Hq + 2 * Hkv, d)[:, Hq + Hkv:]
    page, slot = (t[..., 0] for t in _rows(s, s["len"].long()[..., None] - 1))
    head = torch.arange(Hkv, device=q.device).expand(B, Hkv)
    s["K"][page, slot, head] = k
    s["V"][page, slot, head] = v
    return q


def _attend(s, q, weigh):
    Hq, Hkv, d, B = (s["case"][k] for k in ("Hq", "Hkv", "d", "B"))
    n = s["table"].shape[1] * s["case"]["page"]
    K = s["K"][s["table"].long()].view(B, n, Hkv, d).permute(0, 2, 3, 1).float()
    seen = (torch.arange(n, device=q.device) < s["len"][:, :, None])[:, :, None]
    p = torch.matmul(q.view(B, Hkv, Hq // Hkv, d).float(), K) * (1.0 / math.sqrt(d))
    del K
    p = p.masked_fill(~seen, -math.inf)
    p = torch.exp(p - p.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    V = s["V"][s["table"].long()].view(B, n, Hkv, d).permute(0, 2, 1, 3).float()
    out = torch.matmul(p, V).view(B, Hq, d).bfloat16()
    if weigh:
        s["weights"] += p.sum(2)
    return out


def _evict(s):
    w, c, budget, B, Hkv = (s["case"][k] for k in ("w", "c", "budget", "B", "Hkv"))
    W, n = s["weights"], s["len"].long()[..., None]
    cap = W.shape[2]
    row = torch.arange(cap, device=W.device)
    over = n > budget
    C = torch.where(over, (n - w) // c, 0)                           # chunks that may go
    r = torch.where(over, n - C * c, n)
    k = torch.where(over, (budget - r) // c, 0)
    most = -(-cap // c)
    x = torch.nn.functional.pad(W.double(), (0, most * c - cap)).view(B, Hkv, most, c).sum(-1).float()
    chunk = torch.arange(most, device=W.device)
    x = x.masked_fill(chunk >= C, -math.inf)
    rank = x.argsort(dim=-1, descending=True, stable=True).argsort(dim=-1)   # 0: the largest; equal ones in the order of chunks
    kept = (rank < k) & (chunk < C)
    away, free = kept & (chunk >= k), ~kept & (chunk < k)
    # the j-th kept chunk at or above k goes to the j-th free place below it
    src = chunk.expand(B, Hkv, most).clone()
    at = torch.where(free, free.long().cumsum(-1) - 1, most)
    order = (~away).long().argsort(dim=-1, stable=True)           # the kept ones above k first
    src = torch.where(free, order.gather(-1, at.clamp(max=most - 1)), src)
    new = torch.where(over, k * c + r, n)
    old = src.gather(-1, (row // c).expand(B, Hkv, cap).clamp(max=most - 1)) * c + row % c
    old = torch.where(row < k * c, old, row - k * c + C * c)         # the rows that always stay follow
    old = torch.where(row < new, old, -1)
    sel = (row < new) & (old != row)
    b, h = (torch.arange(m, device=W.device).view(v).expand(B, Hkv, cap) for m, v in ((B, (B, 1, 1)), (Hkv, (1, Hkv, 1))))
    frm, to = _rows(s, old.clamp(min=0)), _rows(s, row.expand(B, Hkv, cap))
    frm, to, h = tuple(t[sel] for t in frm), tuple(t[sel] for t in to), h[sel]
    for cache in (s["K"], s["V"]):
        cache[to[0], to[1], h] = cache[frm[0], frm[1], h]
    W.copy_(torch.where(row < new, W.gather(-1, old.clamp(min=0)), torch.where(row < n, 0.0, W)))
    s["len"].copy_(new[..., 0])
    idx = torch.full((B, Hkv, budget), -1, dtype=torch.int32, device=W.device)
    m = min(budget, cap)
    idx[..., :m] = old[..., :m].int()
    return idx


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    if own:
        import paper_2502_00299_b200 as ck
    case = s["case"]
    kind, Hq, Hkv, d = (case[k] for k in ("kind", "Hq", "Hkv", "d"))
    if kind == "rotate":
        if own:
            return ck.rotate_qk(s["qkv"], Hq, Hkv, d, s["cos"], s["sin"], s["pos"], s["gq"], s["gk"], EPS)
        return _rotate(s)
    if kind == "append":
        if own:
            q = ck.append_paged(s["qkv"], Hq, s["cos"], s["sin"], s["pos"], s["table"], s["len"], s["K"], s["V"], s["gq"], s["gk"], EPS)
        else:
            q = _append(s)
        return q, s["K"], s["V"]
    if kind == "attend":
        return ck.attend_paged(s["q"], s["table"], s["len"], s["K"], s["V"]) if own else _attend(s, s["q"], False)
    if kind == "weigh":
        if own:
            out = ck.attend_paged(s["q"], s["table"], s["len"], s["K"], s["V"], s["weights"])
        else:
            out = _attend(s, s["q"], True)
        return out, s["weights"]
    if kind == "step":
        if own:
            q = ck.append_paged(s["qkv"], Hq, s["cos"], s["sin"], s["pos"], s["table"], s["len"], s["K"], s["V"], s["gq"], s["gk"], EPS)
            out = ck.attend_paged(q, s["table"], s["len"], s["K"], s["V"], s["weights"])
        else:
            q = _append(s)
            out = _attend(s, q, True)
        return q, out, s["weights"], s["K"], s["V"]
    # the sums and lengths that the steps before would have left
    s["weights"].copy_(s["weights0"])
    s["len"].copy_(s["len0"])
    if own:
        idx = ck.evict_paged(s["weights"], s["table"], s["len"], s["K"], s["V"], case["w"], case["c"], case["budget"])
    else:
        idx = _evict(s)
    return idx, s["len"], s["weights"], s["K"], s["V"]


def work(case):
    Hq, Hkv, d, B, L, kind = (case[k] for k in ("Hq", "Hkv", "d", "B", "L", "kind"))
    if kind == "rotate":
        return {"bytes": L * ((Hq + Hkv) * d * 4 + d * 4), "flops": 10 * L * (Hq + Hkv) * d}
    rows = sum(map(sum, _lengths(case)))
    append = {"bytes": B * ((Hq + 2 * Hkv) * d * 4 + d * 4), "flops": 10 * B * (Hq + Hkv) * d}
    if kind == "append":
        return append
    if kind == "evict":
        w, c, budget = (case[k] for k in ("w", "c", "budget"))
        total = 0
        for n in (n for heads in _lengths(case) for n in heads):
            total += 4 * budget
            if n > budget:
                C = (n - w) // c
                r = n - C * c
                k = (budget - r) // c
                total += 4 * n + 2 * ((C - k) * k // max(C, 1) * c + r) * (4 * d + 4)
        return {"bytes": total, "flops": 0}
    got = {"bytes": rows * d * 4 + B * Hq * d * 4 + (rows * 8 if kind in ("weigh", "step") else 0), "flops": 4 * rows * (Hq // Hkv) * d}
    return {k: got[k] + append[k] for k in got} if kind == "step" else got


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_turned(x, gain, cos, sin):
    x = x.to(torch.float64)
    if gain is not None:
        x = x / torch.sqrt(torch.square(x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * gain.to(torch.float64)
    half = x.shape[-1] // 2
    z = torch.complex(x[..., :half], x[..., half:]) * torch.complex(cos.double(), sin.double())[:, None, :]
    return torch.cat((z.real, z.imag), -1)


def _exact_append(s):
    """The token's queries in 64 bits, and the caches with its rows, rounded as they are kept."""
    case = s["case"]
    Hq, Hkv, d, page = (case[k] for k in ("Hq", "Hkv", "d", "page"))
    x = s["qkv"].unflatten(1, (-1, d))
    cos, sin = s["cos"][s["pos"].long()], s["sin"][s["pos"].long()]
    q = _exact_turned(x[:, :Hq], s["gq"], cos, sin)
    k = _exact_turned(x[:, Hq:Hq + Hkv], s["gk"], cos, sin)
    K, V = s["K"].double(), s["V"].double()
    for b, heads in enumerate(s["len"].tolist()):
        for h, n in enumerate(heads):
            p = int(s["table"][b, (n - 1) // page])
            K[p, (n - 1) % page, h] = k[b, h]
            V[p, (n - 1) % page, h] = x[b, Hq + Hkv + h].double()
    return q, K, V


def _exact_attend(s, q, K, V):
    case = s["case"]
    Hkv, d, B, G = case["Hkv"], case["d"], case["B"], case["Hq"] // case["Hkv"]
    out = torch.zeros(B, case["Hq"], d, dtype=torch.float64, device=q.device)
    sums = s["weights"].double() if "weights" in s else None
    for b, heads in enumerate(s["len"].tolist()):
        t = s["table"][b].long()
        Kb, Vb = K[t].flatten(0, 1), V[t].flatten(0, 1)
        for h, n in enumerate(heads):
            z = q[b, h * G:(h + 1) * G].double() @ Kb[:n, h].double().t() / math.sqrt(d)
            p = torch.softmax(z, -1)
            out[b, h * G:(h + 1) * G] = p @ Vb[:n, h].double()
            if sums is not None:
                sums[b, h, :n] += p.sum(0)
    return out, sums


def _exact_evict(s):
    case = s["case"]
    w, c, budget, page = (case[k] for k in ("w", "c", "budget", "page"))
    idx = torch.full((case["B"], case["Hkv"], budget), -1, dtype=torch.int32)
    lens, sums = s["len0"].cpu(), s["weights0"].double().cpu()
    K, V = s["K"].clone(), s["V"].clone()
    for b in range(case["B"]):
        table = s["table"][b].long().cpu()
        for h in range(case["Hkv"]):
            n = int(lens[b, h])
            rows = list(range(n))
            if n > budget:
                C = (n - w) // c
                k = (budget - (n - C * c)) // c
                x = sums[b, h, : C * c].view(C, c).sum(1).float().tolist()
                best = set(sorted(range(C), key=lambda i: (-x[i], i))[:k])
                movers = iter(sorted(i for i in best if i >= k))
                place = [i if i in best else next(movers) for i in range(k)]
                rows = [i * c + j for i in place for j in range(c)] + list(range(C * c, n))
                now = torch.tensor(rows)
                frm, to = now, torch.arange(len(rows))
                for cache in (K, V):
                    cache[table[to // page].cuda(), (to % page).cuda(), h] = (s["K"] if cache is K else s["V"])[table[frm // page].cuda(), (frm % page).cuda(), h]
                sums[b, h, : len(rows)] = sums[b, h, now].clone()
                sums[b, h, len(rows): n] = 0.0
                lens[b, h] = len(rows)
            idx[b, h, : len(rows)] = torch.tensor(rows, dtype=torch.int32)
    return idx, lens, sums, K, V


def exact(case, seed):
    s = prepare(case, seed)
    kind, Hq, Hkv, d = (case[k] for k in ("kind", "Hq", "Hkv", "d"))
    if kind == "rotate":
        x = s["qkv"].unflatten(1, (-1, d))
        cos, sin = s["cos"][s["pos"].long()], s["sin"][s["pos"].long()]
        return _exact_turned(x[:, :Hq], s["gq"], cos, sin), _exact_turned(x[:, Hq:Hq + Hkv], s["gk"], cos, sin)
    if kind == "append":
        return _exact_append(s)
    if kind == "attend":
        return _exact_attend(s, s["q"], s["K"], s["V"])[0]
    if kind == "weigh":
        return _exact_attend(s, s["q"], s["K"], s["V"])
    if kind == "step":
        # attention reads the rows as the cache keeps them, in 16 bits, and so the queries that it is given
        q, K, V = _exact_append(s)
        out, sums = _exact_attend(s, q.bfloat16(), K.bfloat16(), V)
        return q, out, sums, K, V
    return _exact_evict(s)
