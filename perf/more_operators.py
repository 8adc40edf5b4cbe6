"""What a program does with the compacted cache beyond single tokens, as cases that can be timed: tables of rotary angles for long
contexts, queries and keys rotated in either layout, a turn's tokens appended to a paged cache, their attention over it (or to an
encoder's states kept there), and attention of a batch whose sequences share a long prefix.

``own`` false: plain torch operations in 32 bits (angles in 64). ``own`` true: the library's calls.
"""
import math

import torch

own = False

# (query heads, KV heads, head dim): a small model, 8B-class and 70B-class grouped-query shapes, odd and wide groups, heads of their own
SHAPES = ((8, 2, 64), (32, 8, 128), (64, 8, 128), (28, 4, 128), (24, 2, 128), (12, 12, 64))
EPS = 1e-6
POSITIONS = 1 << 17          # rows of the angle tables
BASE = 500000.0
LOGITS = 1 << 30             # of a drawn case, with those of absent rows: what the plain form holds at once


def _case(kind, name=None, Hq=32, Hkv=8, d=128, rot=None, B=1, n=1, L=1, own_rows=0, groups=1, page=16, norm=False, inter=False, ragged=False,
          causal=True, scaling="none", factor=1.0):
    case = dict(kind=kind, Hq=Hq, Hkv=Hkv, d=d, rot=rot or d, B=B, n=n, L=L, own_rows=own_rows, groups=groups, page=page, norm=norm, inter=inter,
                ragged=ragged, causal=causal, scaling=scaling, factor=factor)
    return case if name is None else dict(case, name=name)


def listed():
    return [
        # the tables of a small model that turns half of each head
        _case("rope", "rope 4k x 32", d=64, rot=32, n=4096),
        # tables for a context eight times as long as the one trained on
        _case("rope", "rope 128k x 128", n=131072, scaling="dims", factor=8.0),
        # queries and keys of a prompt's layer before it is compressed: half of each head, neighbours as pairs
        _case("rotate", "rotate 1.5k part", Hq=8, Hkv=2, d=64, rot=32, n=1537, inter=True),
        # the same of a 16K document, whole heads, each normalised
        _case("rotate", "rotate 16k pairs", n=16384, inter=True, norm=True),
        # a short answer typed by one user of a small model
        _case("append", "append 1 x 37", Hq=8, Hkv=2, d=64, rot=32, n=37, L=911),
        # turns of a batch of a 70B-class model
        _case("append", "append 16 ragged 512", Hq=64, B=16, n=512, L=1536, ragged=True, norm=True, inter=True),
        # five guessed tokens a sequence are checked at once
        _case("rows", "rows 8 x 5 over 4k", B=8, n=5, L=4161, ragged=True),
        # a user pastes a long text into a conversation
        _case("rows", "rows 4096 over 8k", n=4096, L=8192, page=64),
        # a batch of decoders' prompts and the states of their encoder, every head on its own
        _case("rows", "cross 8 x 448 to 1500", Hq=12, Hkv=12, d=64, B=8, n=448, L=1500, causal=False, ragged=True),
        # four answers sampled from one prompt that was compressed to a tenth
        _case("shared", "shared 4 over 3.3k", B=4, L=3276, own_rows=70),
        # a full batch of questions about one 32K document
        _case("shared", "shared 64 over 32k", B=64, L=32768, own_rows=600, ragged=True),
        # three documents, seven heads a group, own rows as many as theirs
        _case("shared", "shared 3 groups of 8k", Hq=28, Hkv=4, B=23, groups=3, L=8000, own_rows=1500, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of these ranges."""
    kind = rng.choice(("rope", "rotate", "append", "rows", "rows", "rows", "shared", "shared", "shared"))
    Hq, Hkv, d = rng.choice(SHAPES)
    case = _case(kind, Hq=Hq, Hkv=Hkv, d=d, rot=rng.choice((d, d, d // 2, d // 4, 48)), page=rng.choice((8, 16, 16, 32, 64, 100)),
                 norm=rng.random() < 0.5, inter=rng.random() < 0.5, ragged=rng.random() < 0.6)
    if kind == "rope":
        return dict(case, n=_log(rng, 512, 131072), scaling=rng.choice(("none", "linear", "dims", "waves")), factor=rng.choice((2.0, 4.0, 8.0)))
    if kind == "rotate":
        return dict(case, n=min(_log(rng, 64, 16384), 16384 * 40 // (Hq + Hkv)))
    if kind == "append":
        B = _log(rng, 1, 32)
        n = _log(rng, 1, 512)
        return dict(case, B=B, n=max(1, min(n, 8192 // B)), L=n + _log(rng, 16, 1024))
    if kind == "rows":
        B, n = _log(rng, 1, 16), _log(rng, 1, 4096)
        L = _log(rng, 64, 16384)
        n = max(1, min(n, LOGITS // (B * Hq * (L + n))))
        causal = rng.random() < 0.7
        return dict(case, B=B, n=n, L=L + n if causal else L, causal=causal)
    groups = _log(rng, 1, 4)
    B = max(groups, _log(rng, 1, 64))
    L = min(_log(rng, 256, 32768), 32768 * 64 // (B * groups) * 32 // Hq)
    return dict(case, B=B, groups=groups, L=max(64, L), own_rows=_log(rng, 1, 1024))


def _spread(most, i, ragged):
    """The i-th of some sizes up to `most`: all alike, or spread, the first the largest."""
    return most if not ragged or i == 0 else max(1, most - int(0.9 * most * ((i * 0.6180339887) % 1.0)))


def _tokens(case):
    """New tokens of each sequence; one of a ragged batch of five or more has none."""
    return [0 if case["ragged"] and b == 4 else _spread(case["n"], b, case["ragged"]) for b in range(case["B"])]


def _heads(n, Hkv):
    """Rows of each head of a sequence: some kept a clipped chunk."""
    return [max(0, n - (6 if h % 3 == 1 else 0)) for h in range(Hkv)]


def _lengths(case):
    """Rows of each (sequence, head), new tokens included."""
    kind, B, Hkv, ragged = (case[k] for k in ("kind", "B", "Hkv", "ragged"))
    if kind == "shared":                     # (one of a ragged batch has no row of its own yet)
        return [_heads(0 if ragged and b == 5 else _spread(case["own_rows"], b, ragged), Hkv) for b in range(B)]
    n = _tokens(case)
    if not case["causal"]:
        return [_heads(_spread(case["L"], b, ragged), Hkv) for b in range(B)]
    return [[n[b] + r for r in _heads(_spread(case["L"] - case["n"], b, ragged), Hkv)] for b in range(B)]


def _members(case):
    """Sequences of each group: halves, the rest, ... so that groups differ."""
    B, P = case["B"], case["groups"]
    sizes = []
    for p in range(P):
        left = B - sum(sizes) - (P - 1 - p)
        sizes.append(left if p == P - 1 else max(1, left * 5 // 9))
    return sizes


def _prefixes(case):
    return [_heads(_spread(case["L"], p, case["ragged"]), case["Hkv"]) for p in range(case["groups"])]


def _starts(sizes):
    return torch.tensor([sum(sizes[:i]) for i in range(len(sizes) + 1)], device="cuda", dtype=torch.int32)


def _scaling(case):
    """(factor, length trained on, low, high) of the scaled tables."""
    low, high = {"dims": (1.0, 32.0), "waves": (1.0, 4.0)}.get(case["scaling"], (0.0, 0.0))
    return case["factor"], 8192.0, low, high


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    Hq, Hkv, d, rot, B, page, kind = (case[k] for k in ("Hq", "Hkv", "d", "rot", "B", "page", "kind"))
    dev, bf16, i32 = "cuda", torch.bfloat16, torch.int32
    s = {"case": case}

    def rand(*shape, dtype=bf16):
        return torch.randn(*shape, device=dev, generator=g, dtype=dtype)

    if kind == "rope":
        # a model's base and the first position of this part of its context
        s["base"] = 10000.0 * float(1.0 + 49.0 * torch.rand(1, device=dev, generator=g))
        s["first"] = int(torch.randint(0, POSITIONS, (1,), device=dev, generator=g))
        return s
    if kind in ("rotate", "append"):
        T = case["n"] if kind == "rotate" else sum(_tokens(case))
        s["qkv"] = rand(T, (Hq + 2 * Hkv) * d)
        inv = BASE ** (-torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / rot)
        a = torch.arange(POSITIONS, device=dev, dtype=torch.float64)[:, None] * inv
        s["cos"], s["sin"] = a.cos().float(), a.sin().float()
        first = torch.randint(0, POSITIONS - case["n"], (B,), device=dev, generator=g)
        s["gq"] = (1.0 + 0.2 * rand(d).float()).to(bf16) if case["norm"] else None
        s["gk"] = (1.0 + 0.2 * rand(d).float()).to(bf16) if case["norm"] else None
        sizes = [T] if kind == "rotate" else _tokens(case)
        s["pos"] = torch.cat([first[b] + torch.arange(n, device=dev) for b, n in enumerate(sizes)]).to(i32)
        if kind == "rotate":
            return s
    lens = _lengths(case)
    rows = [max(1, max(x)) for x in lens]
    per = -(-max(rows) // page) + 1
    pre = _prefixes(case) if kind == "shared" else []
    per_pre = -(-max(map(max, pre)) // page) if pre else 0
    pages = B * per + len(pre) * per_pre + 3
    order = torch.randperm(pages, device=dev, generator=g).to(i32)
    s["table"] = order[: B * per].view(B, per).contiguous()
    s["len"] = torch.tensor(lens, device=dev, dtype=i32)
    s["K"], s["V"] = rand(pages, page, Hkv, d), rand(pages, page, Hkv, d)
    if kind == "append":
        s["starts"] = _starts(_tokens(case))
        return s
    # the keys of some rows lie along a direction that their queries share, so that attention is spread unevenly
    u = torch.nn.functional.normalize(rand(Hkv, d, dtype=torch.float32), dim=-1)
    s["K"] += (0.5 * math.sqrt(d) * rand(pages, page, Hkv, 1)) * u.to(bf16)
    T = B if kind == "shared" else sum(_tokens(case))
    s["q"] = (rand(T, Hkv, Hq // Hkv, d, dtype=torch.float32) + 4.0 * u[:, None]).to(bf16).view(T, Hq, d)
    s["starts"] = _starts(_members(case) if kind == "shared" else _tokens(case))
    if pre:
        s["pre_table"] = order[B * per: B * per + len(pre) * per_pre].view(len(pre), per_pre).contiguous()
        s["pre_len"] = torch.tensor(pre, device=dev, dtype=i32)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _frequencies(rot, base, scaling, factor, original, low, high, device):
    i = torch.arange(rot // 2, device=device, dtype=torch.float64)
    inv = base ** (-2.0 * i / rot)
    if scaling == "linear":
        return inv / factor
    if scaling == "dims":        # dims that turn more than `high` times over the length trained on stay, those under `low` times are stretched
        first = max(math.floor(rot * math.log(original / (2.0 * math.pi * high)) / (2.0 * math.log(base))), 0)
        last = min(math.ceil(rot * math.log(original / (2.0 * math.pi * low)) / (2.0 * math.log(base))), rot - 1)
        ramp = ((i - first) / max(last - first, 1e-3)).clamp(0.0, 1.0)
        return inv / factor * ramp + inv * (1.0 - ramp)
    if scaling == "waves":       # the same by wavelengths
        keep = ((original * inv / (2.0 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        return inv / factor * (1.0 - keep) + inv * keep
    return inv


def _rope(s):
    case = s["case"]
    scale = 0.1 * math.log(case["factor"]) + 1.0
    inv = _frequencies(case["rot"], s["base"], case["scaling"], *_scaling(case), "cuda")
    a = (s["first"] + torch.arange(case["n"], device="cuda", dtype=torch.float64))[:, None] * inv
    return (scale * a.cos()).float(), (scale * a.sin()).float()


def _turn(x, gain, cos, sin, inter):
    """x [n, H, d] in 32 bits, cos and sin [n, 1, rot / 2]: the first rot dims turned."""
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()
    rot = 2 * cos.shape[-1]
    y, rest = x[..., :rot], x[..., rot:]
    a, b = (y[..., 0::2], y[..., 1::2]) if inter else y.chunk(2, -1)
    a, b = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((a, b), -1).flatten(-2) if inter else torch.cat((a, b), -1)
    return torch.cat((y, rest), -1)


def _rotate(s):
    Hq, Hkv, d, inter = (s["case"][k] for k in ("Hq", "Hkv", "d", "inter"))
    x = s["qkv"].view(-1, Hq + 2 * Hkv, d)
    cos, sin = s["cos"][s["pos"].long()][:, None], s["sin"][s["pos"].long()][:, None]
    q = _turn(x[:, :Hq].float(), s["gq"], cos, sin, inter)
    k = _turn(x[:, Hq:Hq + Hkv].float(), s["gk"], cos, sin, inter)
    return q.bfloat16(), k.bfloat16()


def _of_tokens(starts, T):
    """(sequence, place within it) of every token."""
    t = torch.arange(T, device=starts.device)
    b = torch.searchsorted(starts[1:].contiguous(), t.to(starts.dtype), right=True)
    return b, t - starts.long()[b]


def _append(s):
    Hq, Hkv, d, page = (s["case"][k] for k in ("Hq", "Hkv", "d", "page"))
    q, k = _rotate(s)
    T = q.shape[0]
    v = s["qkv"].view(T, Hq + 2 * Hkv, d)[:, Hq + Hkv:]
    b, i = _of_tokens(s["starts"], T)
    n = (s["starts"][1:] - s["starts"][:-1]).long()[b]
    row = s["len"].long()[b] - (n - i)[:, None]
    at = s["table"].long()[b[:, None], row // page]
    head = torch.arange(Hkv, device=q.device).expand(T, Hkv)
    s["K"][at, row % page, head] = k
    s["V"][at, row % page, head] = v
    return q


def _scores(q, K, table, seen):
    """q [sets, tokens, Hq, d] over the rows of their tables: maximum, sum and numerator in 32 bits. seen [sets, Hkv, tokens, rows]."""
    S, n, Hq, d = q.shape
    Kg, V = K
    Hkv = Kg.shape[2]
    rows = table.shape[1] * Kg.shape[1]
    k = Kg[table.long()].view(S, rows, Hkv, d).permute(0, 2, 3, 1).float()
    x = q.view(S, n, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4).reshape(S, Hkv, -1, d).float()
    p = torch.matmul(x, k).mul_(1.0 / math.sqrt(d)).view(S, Hkv, Hq // Hkv, n, rows)
    p.masked_fill_(~seen[:, :, None], -math.inf)
    m = p.amax(-1, keepdim=True)
    p = p.sub_(m.clamp(min=-3e38)).exp_()
    l = p.sum(-1, keepdim=True)
    v = V[table.long()].view(S, rows, Hkv, d).permute(0, 2, 1, 3).float()
    o = torch.matmul(p.view(S, Hkv, -1, rows), v).view(S, Hkv, Hq // Hkv, n, d)
    return tuple(t.permute(0, 3, 1, 2, 4).reshape(S, n, Hq, -1) for t in (m, l, o))


def _rows(s):
    case = s["case"]
    T, Hq, d = s["q"].shape
    n = max(case["n"], 1)
    b, i = _of_tokens(s["starts"], T)
    q = torch.zeros(case["B"], n, Hq, d, device="cuda", dtype=s["q"].dtype)
    q[b, i] = s["q"]
    row = torch.arange(s["table"].shape[1] * case["page"], device="cuda")
    limit = s["len"].long()[:, :, None]
    if case["causal"]:
        count = (s["starts"][1:] - s["starts"][:-1]).long()
        limit = limit - count[:, None, None] + 1 + torch.arange(n, device="cuda")
    m, l, o = _scores(q, (s["K"], s["V"]), s["table"], row < limit.expand(-1, -1, n)[..., None])
    out = o / l.clamp(min=1e-30)
    return out[b, i].bfloat16()


def _shared(s):
    case = s["case"]
    B, Hq, d = s["q"].shape
    g, i = _of_tokens(s["starts"], B)
    most = max(_members(case))
    q = torch.zeros(case["groups"], most, Hq, d, device="cuda", dtype=s["q"].dtype)
    q[g, i] = s["q"]
    parts = []
    for x, table, lens in ((q, s["pre_table"], s["pre_len"]), (s["q"][:, None], s["table"], s["len"])):
        row = torch.arange(table.shape[1] * case["page"], device="cuda")
        seen = (row < lens.long()[:, :, None])[:, :, None].expand(-1, -1, x.shape[1], -1)
        parts.append(_scores(x, (s["K"], s["V"]), table, seen))
    (m0, l0, o0), (m1, l1, o1) = [t[g, i] for t in parts[0]], [t[:, 0] for t in parts[1]]
    m = torch.maximum(m0, m1).clamp(min=-3e38)
    f0, f1 = torch.exp(m0 - m), torch.exp(m1 - m)
    return ((o0 * f0 + o1 * f1) / (l0 * f0 + l1 * f1).clamp(min=1e-30)).bfloat16()


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    if own:
        import paper_2502_00299_b200 as ck
    case = s["case"]
    kind, Hq, Hkv, d, inter = (case[k] for k in ("kind", "Hq", "Hkv", "d", "inter"))
    if kind == "rope":
        if own:
            factor, original, low, high = _scaling(case)
            return ck.rope_tables(case["n"], case["rot"], s["base"], case["scaling"], factor, original, low, high,
                                  scale=0.1 * math.log(factor) + 1.0, first=s["first"])
        return _rope(s)
    if kind == "rotate":
        if own:
            return ck.rotate_rows(s["qkv"], Hq, Hkv, d, s["cos"], s["sin"], s["pos"], inter, s["gq"], s["gk"], EPS)
        return _rotate(s)
    if kind == "append":
        if own:
            q = ck.append_rows_paged(s["qkv"], Hq, s["starts"], s["cos"], s["sin"], s["pos"], s["table"], s["len"], s["K"], s["V"], inter,
                                     s["gq"], s["gk"], EPS)
        else:
            q = _append(s)
        return q, s["K"], s["V"]
    if kind == "rows":
        if own:
            return ck.attend_rows_paged(s["q"], s["starts"], s["table"], s["len"], s["K"], s["V"], case["causal"])
        return _rows(s)
    if own:
        return ck.attend_shared_paged(s["q"], s["starts"], s["pre_table"], s["pre_len"], s["table"], s["len"], s["K"], s["V"])
    return _shared(s)


def work(case):
    kind, Hq, Hkv, d, rot, B = (case[k] for k in ("kind", "Hq", "Hkv", "d", "rot", "B"))
    if kind == "rope":
        return {"bytes": 4 * case["n"] * rot, "flops": 20 * case["n"] * rot}
    if kind == "rotate":
        return {"bytes": case["n"] * ((Hq + Hkv) * d * 4 + rot * 4), "flops": 10 * case["n"] * (Hq + Hkv) * d}
    if kind == "append":
        T = sum(_tokens(case))
        return {"bytes": T * ((Hq + 2 * Hkv) * d * 4 + rot * 4), "flops": 10 * T * (Hq + Hkv) * d}
    lens, G = _lengths(case), Hq // Hkv
    if kind == "rows":
        n = _tokens(case)
        seen = sum(sum(max(0, x - (n[b] - 1 - i) if case["causal"] else x) for i in range(n[b])) for b in range(B) for x in lens[b])
        rows = sum(x for b in range(B) for x in lens[b] if n[b])
        return {"bytes": rows * d * 4 + sum(n) * Hq * d * 4, "flops": 4 * seen * G * d}
    pre = _prefixes(case)
    rows = sum(map(sum, lens)) + sum(map(sum, pre))
    seen = sum(map(sum, lens)) + sum(m * sum(x) for m, x in zip(_members(case), pre))
    return {"bytes": rows * d * 4 + B * Hq * d * 4, "flops": 4 * seen * G * d}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_rope(s):
    case = s["case"]
    rot, base, f = case["rot"], s["base"], case["factor"]
    inv = []
    for i in range(rot // 2):
        w = base ** (-2.0 * i / rot)
        if case["scaling"] == "linear":
            w /= f
        elif case["scaling"] == "dims":
            at = [rot * math.log(8192.0 / (turns * 2.0 * math.pi)) / (2.0 * math.log(base)) for turns in (32.0, 1.0)]
            first, last = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
            part = min(max((i - first) / max(last - first, 1e-3), 0.0), 1.0)
            w = w * (1.0 - part) + w / f * part
        elif case["scaling"] == "waves":
            wave = 2.0 * math.pi / w
            if wave > 8192.0 / 1.0:
                w /= f
            elif wave >= 8192.0 / 4.0:
                part = (8192.0 / wave - 1.0) / (4.0 - 1.0)
                w = (1.0 - part) * w / f + part * w
        inv.append(w)
    p = torch.arange(s["first"], s["first"] + case["n"], device="cuda", dtype=torch.float64)
    z = torch.polar(torch.tensor(1.0 + 0.1 * math.log(f), device="cuda", dtype=torch.float64).expand(case["n"], rot // 2),
                    p[:, None] * torch.tensor(inv, device="cuda", dtype=torch.float64))
    return z.real, z.imag


def _exact_turned(x, gain, cos, sin, inter):
    x = x.to(torch.float64)
    if gain is not None:
        x = x / torch.sqrt(torch.square(x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * gain.to(torch.float64)
    h = cos.shape[1]
    x = x.clone()
    first = slice(0, 2 * h, 2) if inter else slice(0, h)
    second = slice(1, 2 * h, 2) if inter else slice(h, 2 * h)
    z = torch.complex(x[..., first].clone(), x[..., second].clone()) * torch.complex(cos.double(), sin.double())[:, None, :]
    x[..., first], x[..., second] = z.real, z.imag
    return x


def _exact_qk(s):
    case = s["case"]
    Hq, Hkv, d = (case[k] for k in ("Hq", "Hkv", "d"))
    x = s["qkv"].unflatten(1, (-1, d))
    cos, sin = s["cos"][s["pos"].long()], s["sin"][s["pos"].long()]
    q = _exact_turned(x[:, :Hq], s["gq"], cos, sin, case["inter"])
    return q, _exact_turned(x[:, Hq:Hq + Hkv], s["gk"], cos, sin, case["inter"]), x[:, Hq + Hkv:].double()


def _exact_append(s):
    case = s["case"]
    Hkv, page = case["Hkv"], case["page"]
    q, k, v = _exact_qk(s)
    K, V = s["K"].double(), s["V"].double()
    first = s["starts"].tolist()
    for b, heads in enumerate(s["len"].tolist()):
        n = first[b + 1] - first[b]
        for h, end in enumerate(heads):
            rows = torch.arange(end - n, end, device="cuda")
            at = s["table"][b].long()[rows // page]
            K[at, rows % page, h] = k[first[b]: first[b + 1], h]
            V[at, rows % page, h] = v[first[b]: first[b + 1], h]
    return q, K, V


def _exact_heads(s, table, h, n):
    """Keys and values of a head's first n rows in 64 bits."""
    page = s["case"]["page"]
    rows = torch.arange(n, device="cuda")
    at = table.long()[rows // page]
    return s["K"][at, rows % page, h].double(), s["V"][at, rows % page, h].double()


def _exact_rows(s):
    case = s["case"]
    Hkv, d, G = case["Hkv"], case["d"], case["Hq"] // case["Hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    first = s["starts"].tolist()
    for b, heads in enumerate(s["len"].tolist()):
        n = first[b + 1] - first[b]
        for h, L in enumerate(heads):
            K, V = _exact_heads(s, s["table"][b], h, L)
            for g in range(h * G, (h + 1) * G):
                z = s["q"][first[b]: first[b + 1], g].double() @ K.t() / math.sqrt(d)
                if case["causal"]:
                    z += torch.full_like(z, -math.inf).triu(L - n + 1)
                if L and n:
                    out[first[b]: first[b + 1], g] = torch.softmax(z, -1).nan_to_num(0.0) @ V
    return out


def _exact_shared(s):
    case = s["case"]
    Hkv, d, G = case["Hkv"], case["d"], case["Hq"] // case["Hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    first, pre, own_rows = s["starts"].tolist(), s["pre_len"].tolist(), s["len"].tolist()
    for p in range(case["groups"]):
        for h in range(Hkv):
            K, V = _exact_heads(s, s["pre_table"][p], h, pre[p][h])
            for b in range(first[p], first[p + 1]):
                k, v = _exact_heads(s, s["table"][b], h, own_rows[b][h])
                q = s["q"][b, h * G:(h + 1) * G].double()
                z = torch.cat((q @ K.t(), q @ k.t()), 1) / math.sqrt(d)
                z = torch.softmax(z, -1)
                out[b, h * G:(h + 1) * G] = z[:, :len(K)] @ V + z[:, len(K):] @ v
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rope":
        return _exact_rope(s)
    if kind == "rotate":
        return _exact_qk(s)[:2]
    if kind == "append":
        return _exact_append(s)
    return _exact_rows(s) if kind == "rows" else _exact_shared(s)
