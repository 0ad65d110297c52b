"""Cases of the operators around a caller-owned, paged K/V store of eight bits, beside `wnw_attend_static`.

Five kinds of case.

`rotate`  rotary positions with several axes for the queries and keys of a layer, or, inverse, for their gradients
          (`wnw_rotate`).
`write`   new K,V rows of a ragged batch, quantised as they enter the pages (`wnw_pages_write`).
`read`    a run of tokens of each sequence, read back from the pages (`wnw_pages_read`).
`attend`  attention of a ragged batch of query rows over the pages (`wnw_pages_attend`).
`step`    the three of them as a decoder's layer uses them for one token of every sequence: rotate the queries, rotate and
          write the new key, write the new value, attend.

The store: codes [pages][kv_heads][K|V][page_tokens][dim], one byte each, and one power-of-two scale for each page, head and
K|V: 2^e with e the integer that brings the largest magnitude of the block's rows into (224, 448] (e4m3) or (63.5, 127]
(int8), -110 for rows of zeros only.  A write into a page that holds rows already keeps its scale or raises it; a raise rounds
the codes held anew.
"""
import math

import torch

own = False

REGION = 64       # tokens that share one direction in the synthetic keys
E4M3, INT8 = "e4m3", "int8"
LARGEST = {E4M3: 448.0, INT8: 127.0}
HIGHEST = {E4M3: 119, INT8: 121}      # of the scales' exponents
LOWEST = -110
DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _case(kind, name=None, **changes):
    case = dict(kind=kind, q_heads=32, kv_heads=8, dim=128, dtype="bf16")
    if kind != "rotate":
        case.update(format=E4M3, page=64, seqs=1, tokens=3064, ragged=False)
    if kind in ("rotate", "step"):
        case.update(base=1e6, axes=3, dealt=False, neighbours=False)
    if kind == "rotate":
        case.update(tokens=64, inverse=False, fused=False)
    if kind == "write":
        case.update(rows=1)
    if kind == "attend":
        case.update(rows=1, causal=True, lse=False)
    case.update(changes)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # one token of each of a few requests: launch and host latency
        _case("rotate", "rotate_token", tokens=4, q_heads=16, kv_heads=2),
        # the gradient of a whole prompt's queries and keys, slices of the projection's output: ten minutes of audio with its text
        _case("rotate", "rotate_prompt_back", tokens=15064, q_heads=16, kv_heads=2, inverse=True, fused=True),
        # a token of each of 32 requests enters its last page
        _case("write", "write_token", seqs=32, tokens=7500, ragged=True),
        # the prompts of four requests, up to ten minutes each
        _case("write", "write_prompt", format=INT8, seqs=4, tokens=0, rows=15001, ragged=True),
        # a four-minute clip comes back for another request
        _case("read", "read_clip", tokens=3064),
        # an hour of audio comes back as fp16
        _case("read", "read_hour", tokens=50001, format=INT8, dtype="fp16"),
        # the smallest attention: one token of a small model over half a minute of audio
        _case("attend", "attend_short", q_heads=8, kv_heads=4, dim=64, tokens=777, page=32, lse=True),
        # one token of a request of four minutes
        _case("attend", "attend_clip", tokens=3064),
        # one token of each of 32 requests of different lengths
        _case("attend", "attend_batch", seqs=32, tokens=7500, ragged=True, format=INT8, lse=True),
        # one token of 16 hour-long requests: the largest store
        _case("attend", "attend_hours", seqs=16, tokens=50001),
        # a piece of a long prompt, behind what has been written of it
        _case("attend", "attend_prompt", tokens=15064, rows=2049),
        # one token of a layer, everything that touches the store
        _case("step", "step_batch", seqs=16, q_heads=16, kv_heads=2, tokens=15000, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    limit = {}
    for c in listed():
        w = work(c)
        top = limit.setdefault(c["kind"], [0, 0])
        limit[c["kind"]] = [max(top[0], w["bytes"]), max(top[1], w["flops"])]
    limit["step"] = limit["attend"]
    while True:
        case = _draw(rng)
        w = work(case)
        if w["bytes"] <= limit[case["kind"]][0] and w["flops"] <= limit[case["kind"]][1]:
            return case


def _draw(rng):
    kind = rng.choice(["rotate", "write", "read", "attend", "attend", "attend", "step"])
    q_heads, kv_heads, dim = rng.choice([(8, 4, 64), (32, 8, 128), (32, 8, 128), (16, 2, 128), (16, 4, 64), (5, 5, 64), (28, 4, 128), (20, 2, 64)])
    case = _case(kind, q_heads=q_heads, kv_heads=kv_heads, dim=dim, dtype=rng.choice(["bf16", "bf16", "fp16"]))
    if kind in ("rotate", "step"):
        case.update(base=rng.choice([1e4, 1e6]), axes=rng.choice([1, 2, 3]), dealt=rng.random() < 0.5, neighbours=rng.random() < 0.3)
    if kind == "rotate":
        case.update(tokens=_log_int(rng, 1, 15064), inverse=rng.random() < 0.5, fused=rng.random() < 0.5)
        if rng.random() < 0.2:
            case.update(dtype="fp32")
        return case
    case.update(page=rng.choice([16, 32, 48, 64, 64, 128]), ragged=rng.random() < 0.6)
    if kind != "step":     # a rounding of the rotated key may move an eight-bit integer: the step is drawn in e4m3
        case.update(format=rng.choice([E4M3, E4M3, INT8]))
    if kind == "write":
        prompt = rng.random() < 0.5
        case.update(seqs=_log_int(rng, 1, 8 if prompt else 96), rows=_log_int(rng, 17, 15001) if prompt else rng.randint(1, 5),
                    tokens=_log_int(rng, 1, 9000) if rng.random() < 0.8 else 0)
    elif kind == "read":
        case.update(seqs=_log_int(rng, 1, 8), tokens=_log_int(rng, 1, 50001))
    elif kind == "attend":
        rows = rng.choice([1, 1, 1, rng.randint(2, 8), _log_int(rng, 9, 2049)])
        case.update(seqs=_log_int(rng, 1, 64), tokens=max(rows, _log_int(rng, 1, 50001)), rows=rows, causal=rng.random() < 0.8, lse=rng.random() < 0.5)
    else:
        case.update(seqs=_log_int(rng, 1, 64), tokens=_log_int(rng, 1, 15000))
    return case


# ---------------------------------------------------------------------------------------------------------------- shapes
def _ragged(n, count, salt):
    """`count` lengths up to n: the first is n, the others anything from a quarter of it on."""
    g = torch.Generator().manual_seed(8191 * n + 31 * count + salt)
    low = (n + 3) // 4
    return [n] + [int(x) for x in torch.randint(low, n + 1, (count - 1,), generator=g)] if count > 1 else [n]


def _shape(case):
    """(tokens held before the call, rows of the call) of every sequence.  `read`: the first token read, and how many."""
    seqs = case["seqs"]
    lengths = _ragged(case["tokens"], seqs, 1) if case["ragged"] else [case["tokens"]] * seqs
    if case["kind"] == "read":
        begins = [min(7 * b, n - 1) for b, n in enumerate(lengths)]
        return begins, [n - a for a, n in zip(begins, lengths)]
    if case["kind"] == "step":
        return lengths, [1] * seqs
    rows = _ragged(case["rows"], seqs, 2) if case["ragged"] else [case["rows"]] * seqs
    if case["kind"] == "attend":     # the rows' own keys are in the pages already
        return [max(0, n - r) for n, r in zip(lengths, rows)], rows
    return lengths, rows


def _sections(pairs, axes):
    """Pairs of each axis: the first (time) a quarter, the others the rest in equal shares."""
    if axes == 1:
        return [pairs]
    first = pairs // 4 if axes == 3 else pairs // 2
    rest = (pairs - first) // (axes - 1)
    return [pairs - rest * (axes - 1)] + [rest] * (axes - 1)


def _axis_of_pair(pairs, sections, dealt):
    """The axis that turns each pair: consecutive runs, or dealt in turn (an axis that has had its share leaves its turn to
    the first)."""
    n = len(sections)
    if not dealt:
        return [a for a, s in enumerate(sections) for _ in range(s)]
    return [i % n if i // n < sections[i % n] else 0 for i in range(pairs)]


def work(case):
    q_heads, H, d, size = case["q_heads"], case["kv_heads"], case["dim"], DTYPE[case["dtype"]].itemsize
    if case["kind"] == "rotate":
        n = case["tokens"] * (q_heads + H) * d
        return {"bytes": 2 * n * size + 4 * case["axes"] * case["tokens"], "flops": 3 * n}
    held, rows = _shape(case)
    n_rows, page = sum(rows), case["page"]
    pages = sum((n + r + page - 1) // page - n // page for n, r in zip(held, rows))
    table = 4 * pages + 8 * case["seqs"]
    enter = 2 * n_rows * H * d * (size + 1) + 8 * pages * H + table
    if case["kind"] in ("write", "read"):
        return {"bytes": enter, "flops": 4 * n_rows * H * d}
    causal = case.get("causal", True)
    seen = sum(r * n + (r * (r + 1) // 2 if causal else r * r) for n, r in zip(held, rows))
    every = sum((n + r + page - 1) // page for n, r in zip(held, rows))
    total = 2 * H * d * sum(n + r for n, r in zip(held, rows)) + 8 * every * H + 4 * every + 2 * n_rows * q_heads * d * size
    flops = 4 * q_heads * d * seen
    if case["kind"] == "step":
        total += enter + 2 * n_rows * q_heads * d * size
        flops += 3 * n_rows * (q_heads + H) * d
    elif case["lse"]:
        total += 4 * n_rows * q_heads
    return {"bytes": total, "flops": flops}


# ---------------------------------------------------------------------------------------------------------------- inputs
class _State:
    pass


def _exponent(amax, fmt):
    """The scale's exponent for rows of these largest magnitudes."""
    mantissa, e = torch.frexp(amax)                       # amax = mantissa * 2^e, mantissa in [0.5, 1)
    top, bits = math.frexp(LARGEST[fmt])
    e = e - torch.where(mantissa <= top, bits, bits - 1)
    return torch.where(amax > 0, e, LOWEST).clamp(LOWEST, HIGHEST[fmt])


def _power(e):
    """2^e as float32, exactly (-126 <= e <= 127)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _round(x, fmt):
    """Scaled values to codes, as the numbers that they are (any floating type)."""
    if fmt == INT8:
        return x.round().clamp(-127, 127)
    return x.clamp(-448, 448).to(torch.float32).to(torch.float8_e4m3fn).to(x.dtype)


def _as_codes(x, fmt):
    return x.to(torch.int8 if fmt == INT8 else torch.float8_e4m3fn)


def _fill(s, case, randn, total):
    """Pages that hold `total[b]` tokens of each sequence: keys with a direction for each region of tokens, as audio has."""
    H, d, T, fmt = case["kv_heads"], case["dim"], case["page"], case["format"]
    counts = [(n + T - 1) // T for n in total]
    widest, n_pages = max(counts + [1]), sum(counts) + 3
    perm = torch.randperm(n_pages, generator=s.gen, device="cuda")
    s.table = torch.zeros(len(total), widest, dtype=torch.int32, device="cuda")
    s.codes = torch.empty(n_pages, H, 2, T, d, dtype=torch.int8 if fmt == INT8 else torch.float8_e4m3fn, device="cuda")
    s.scales = torch.empty(n_pages, H, 2, dtype=torch.float32, device="cuda")
    n_regions = widest * T // REGION + 1
    s.directions = 4.0 * torch.nn.functional.normalize(randn(H, n_regions, d, dtype=torch.float32), dim=-1)
    first = 0
    for b, n in enumerate(counts):
        s.table[b, :n] = perm[first:first + n].to(torch.int32)
        first += n
    place = torch.cat([torch.arange(n, device="cuda") for n in counts] + [torch.zeros(3, dtype=torch.long, device="cuda")])
    for at in range(0, n_pages, 2048):
        p = place[at:at + 2048]
        x = randn(len(p), H, 2, T, d, dtype=torch.float32)
        region = (p.unsqueeze(1) * T + torch.arange(T, device="cuda")) // REGION                # [pages][T]
        x[:, :, 0] += s.directions[:, region].transpose(0, 1)
        x = x.to(DTYPE[case["dtype"]]).float()
        e = _exponent(x.abs().amax((3, 4)), fmt)
        s.scales[perm[at:at + 2048]] = _power(e)
        codes = _as_codes(_round(x * _power(-e)[..., None, None], fmt), fmt)
        s.codes.view(torch.uint8)[perm[at:at + 2048]] = codes.view(torch.uint8)


def _positions(s, case, first):
    """[axes][tokens]: time runs on, the other axes lie within an image."""
    n, axes = len(first), case["axes"]
    t = torch.tensor(first, dtype=torch.int32, device="cuda").unsqueeze(0)
    rest = torch.randint(0, 64, (axes - 1, n), generator=s.gen, device="cuda", dtype=torch.int32)
    return torch.cat([t, rest])


def prepare(case, seed):
    s = _State()
    s.case = case
    s.gen = torch.Generator(device="cuda")
    s.gen.manual_seed(seed)
    dtype, Hq, H, d = DTYPE[case["dtype"]], case["q_heads"], case["kv_heads"], case["dim"]

    def randn(*shape, dtype=dtype):
        return torch.randn(*shape, generator=s.gen, device="cuda", dtype=dtype)

    if case["kind"] in ("rotate", "step"):
        pairs = d // 2
        s.sections = _sections(pairs, case["axes"])
        if own:
            import paper_2608_22704_b200 as wnw
            s.rotary = wnw.wnw_rotary_init(pairs, case["base"], s.sections, dealt=case["dealt"], neighbours=case["neighbours"])
        s.frequency = torch.pow(torch.tensor(case["base"], dtype=torch.float64, device="cuda"),
                                -torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)
        s.axis = torch.tensor(_axis_of_pair(pairs, s.sections, case["dealt"]), device="cuda")
    if case["kind"] == "rotate":
        n = case["tokens"]
        if case["fused"]:                                   # slices of one projection's output
            qkv = randn(n, Hq + 2 * H, d)
            s.q, s.k = qkv[:, :Hq], qkv[:, Hq:Hq + H]
        else:
            s.q, s.k = randn(n, Hq, d), randn(n, H, d)
        s.q_out, s.k_out = (torch.empty(x.shape, dtype=dtype, device="cuda") for x in (s.q, s.k))
        s.positions = _positions(s, case, range(100003, 100003 + n))
        return s

    held, rows = _shape(case)
    s.held, s.rows, n_rows = held, rows, sum(rows)
    starts = [0]
    for r in rows:
        starts.append(starts[-1] + r)
    s.row_starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
    s.lengths = torch.tensor(held, dtype=torch.int32, device="cuda")
    s.lengths_after = s.lengths + torch.tensor(rows, dtype=torch.int32, device="cuda")
    s.max_rows = max(rows)
    _fill(s, case, randn, [n + r for n, r in zip(held, rows)])
    if case["kind"] in ("write", "step"):
        s.k, s.v = randn(n_rows, H, d), randn(n_rows, H, d)
    elif case["kind"] == "read":
        s.k, s.v = (torch.empty(n_rows, H, d, dtype=dtype, device="cuda") for _ in range(2))
    if case["kind"] in ("attend", "step"):
        # a query leans on one region of its sequence
        owner = torch.repeat_interleave(torch.arange(len(rows), device="cuda"), torch.tensor(rows, device="cuda"))
        region = (torch.rand(n_rows, generator=s.gen, device="cuda") * s.lengths_after[owner] / REGION).long()
        lean = s.directions[:, region].transpose(0, 1).repeat_interleave(Hq // H, dim=1)
        s.q = (randn(n_rows, Hq, d, dtype=torch.float32) + 0.25 * math.sqrt(d) * lean).to(dtype)
        s.out = torch.zeros(n_rows, Hq, d, dtype=dtype, device="cuda")
        s.lse = torch.zeros(n_rows, Hq, dtype=torch.float32, device="cuda") if case.get("lse") else None
    if case["kind"] == "step":
        s.positions = _positions(s, case, held)
        s.q_rotated = torch.empty_like(s.q)
    del s.directions
    if own:
        import paper_2608_22704_b200 as wnw
        s.pages = wnw.wnw_pages(s.codes, s.scales)
        if case["kind"] in ("attend", "step"):
            s.workspace = torch.empty(wnw.wnw_pages_attend_workspace(s.pages, Hq), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------------------- passes
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2608_22704_b200 as wnw
    case, kind = s.case, s.case["kind"]
    if kind == "rotate":
        wnw.wnw_rotate(s.rotary, s.positions, s.q, s.q_out, s.k, s.k_out, inverse=case["inverse"])
        return s.q_out, s.k_out
    if kind == "write":
        wnw.wnw_pages_write(s.pages, s.table, s.lengths, s.row_starts, s.k, s.v, max_rows=s.max_rows)
        return s.codes, s.scales
    if kind == "read":
        wnw.wnw_pages_read(s.pages, s.table, s.lengths, s.row_starts, s.k, s.v, max_rows=s.max_rows)
        return s.k, s.v
    if kind == "attend":
        wnw.wnw_pages_attend(s.pages, s.table, s.lengths_after, s.row_starts, s.q, s.out, s.workspace, lse=s.lse, causal=case["causal"],
                             max_rows=s.max_rows)
        return (s.out, s.lse) if case["lse"] else s.out
    wnw.wnw_rotate(s.rotary, s.positions, s.q, s.q_rotated)
    wnw.wnw_pages_write(s.pages, s.table, s.lengths, s.row_starts, s.k, s.v, rotary=s.rotary, positions=s.positions, max_rows=1)
    wnw.wnw_pages_attend(s.pages, s.table, s.lengths_after, s.row_starts, s.q_rotated, s.out, s.workspace, max_rows=1)
    return s.out, s.codes, s.scales


def _run_plain(s):
    case, kind = s.case, s.case["kind"]
    if kind == "rotate":
        s.q_out.copy_(_rotate(s, s.q, case["inverse"]))
        s.k_out.copy_(_rotate(s, s.k, case["inverse"]))
        return s.q_out, s.k_out
    if kind == "write":
        _write(s, s.k, s.v)
        return s.codes, s.scales
    if kind == "read":
        _read(s)
        return s.k, s.v
    if kind == "attend":
        _attend(s, s.q, case["causal"])
        return (s.out, s.lse) if case["lse"] else s.out
    q = _rotate(s, s.q, False).to(s.q.dtype)
    _write(s, _rotate(s, s.k, False).to(s.k.dtype), s.v)
    _attend(s, q, True)
    return s.out, s.codes, s.scales


def _rotate(s, x, inverse):
    """x [tokens][heads][dim] turned by its positions, as float32.  Angles of far positions lose what matters in 32 bits: 64."""
    angle = s.positions.double()[s.axis].transpose(0, 1) * s.frequency                       # [tokens][pairs]
    if inverse:
        angle = -angle
    c, sn = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
    x = x.float()
    pairs = s.axis.numel()
    if s.case["neighbours"]:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * c - b * sn, b * c + a * sn], dim=-1).flatten(-2)
    a, b = x[..., :pairs], x[..., pairs:]
    return torch.cat([a * c - b * sn, b * c + a * sn], dim=-1)


def _write(s, k, v):
    """All pages that a call touches at once: [seqs][most pages of a sequence]."""
    case = s.case
    T, fmt = case["page"], case["format"]
    first, last = s.lengths // T, (s.lengths_after + T - 1) // T
    most = max((n + r + T - 1) // T - n // T for n, r in zip(s.held, s.rows))
    at = first.unsqueeze(1) + torch.arange(most, device="cuda")                              # page of the sequence
    seq, nth = (at < last.unsqueeze(1)).nonzero(as_tuple=True)
    at = at[seq, nth]
    page = s.table[seq, at].long()
    token = at.unsqueeze(1) * T + torch.arange(T, device="cuda")                             # [pages][T]
    new = (token >= s.lengths[seq].unsqueeze(1)) & (token < s.lengths_after[seq].unsqueeze(1))
    old = token < s.lengths[seq].unsqueeze(1)
    row = (s.row_starts[seq].unsqueeze(1) + token - s.lengths[seq].unsqueeze(1)) * new
    x = torch.stack([k, v], dim=2)[row].permute(0, 2, 3, 1, 4).float()                       # [pages][heads][K|V][T][dim]
    new, old = new[:, None, None, :, None], old[:, None, None, :, None]
    x = torch.where(new, x, 0.0)
    had = torch.where(old.any(3).squeeze(-1), torch.frexp(s.scales[page])[1] - 1, LOWEST)
    e = torch.maximum(had, _exponent(x.abs().amax((3, 4)), fmt))
    fresh = _round(x * _power(-e)[..., None, None], fmt)
    kept = s.codes[page].float()
    kept = torch.where(old, _round(kept * _power((had - e).clamp(min=-64))[..., None, None], fmt), kept)
    codes = _as_codes(torch.where(new, fresh, kept), fmt)
    s.codes.view(torch.uint8)[page] = codes.view(torch.uint8)
    s.scales[page] = _power(e)


def _read(s):
    T = s.case["page"]
    n = s.row_starts.diff()
    seq = torch.repeat_interleave(torch.arange(len(s.rows), device="cuda"), n)
    token = torch.arange(len(seq), device="cuda") - s.row_starts[seq] + s.lengths[seq]
    page, row = s.table[seq, token // T].long(), token % T
    x = s.codes[page, :, :, row].float() * s.scales[page].unsqueeze(-1)                      # [rows][heads][K|V][dim]
    most = torch.finfo(s.k.dtype).max
    x = x.clamp(-most, most)
    s.k.copy_(x[:, :, 0])
    s.v.copy_(x[:, :, 1])


def _attend(s, q, causal):
    """The batch padded to its longest sequence and its most rows."""
    case = s.case
    H, d, T, B, R = case["kv_heads"], case["dim"], case["page"], len(s.rows), s.max_rows
    group, P = case["q_heads"] // H, s.table.shape[1]
    page = s.table.long()
    x = s.codes[page].float() * s.scales[page][..., None, None]                              # [B][P][H][2][T][d]
    x = x.permute(3, 0, 2, 1, 4, 5).reshape(2, B, H, P * T, d)
    nth = torch.arange(R, device="cuda")
    real = nth < s.row_starts.diff().unsqueeze(1)                                            # [B][R]
    row = (s.row_starts[:-1].unsqueeze(1) + nth) * real
    qs = q[row].float().view(B, R, H, group, d).permute(0, 2, 1, 3, 4).reshape(B, H, R * group, d)
    scores = (qs @ x[0].transpose(-1, -2) / math.sqrt(d)).view(B, H, R, group, P * T)
    token = torch.arange(P * T, device="cuda")
    end = s.lengths_after.unsqueeze(1).expand(B, R)
    if causal:
        end = end - s.row_starts.diff().unsqueeze(1) + nth + 1
    seen = (token < end.unsqueeze(-1))[:, None, :, None]                                     # [B][1][R][1][P*T]
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    e = (scores - top.clamp(min=-1e30)).exp()
    total = e.sum(-1, keepdim=True)
    values = x[1].masked_fill((token >= s.lengths_after.unsqueeze(1))[:, None, :, None], 0.0)
    out = (e.view(B, H, R * group, P * T) @ values).view(B, H, R, group, d) / total.clamp(min=1e-30)
    s.out[row[real]] = out.permute(0, 2, 1, 3, 4).reshape(B, R, H * group, d)[real].to(s.out.dtype)
    if s.lse is not None:
        s.lse[row[real]] = (top + total.log()).squeeze(-1).permute(0, 2, 1, 3).reshape(B, R, H * group)[real]


# ------------------------------------------------------------------------------------------------- definitions in 64 bits
def exact(case, seed):
    """What `run` returns, by the operators' definitions: a sequence, a page and a head at a time."""
    s = prepare(case, seed)
    if case["kind"] == "rotate":
        return [_exact_rotate(s, x, -1.0 if case["inverse"] else 1.0) for x in (s.q, s.k)]
    scales = s.scales.double()
    codes = s.codes.double() if case["kind"] in ("write", "step") else None
    if case["kind"] == "write":
        _exact_write(s, codes, scales, s.k.double(), s.v.double())
        return [None if case["format"] == INT8 else codes, scales]
    if case["kind"] == "read":
        return _exact_read(s, scales)
    if case["kind"] == "attend":
        out, lse = _exact_attend(s, s.codes, scales, s.q.double(), case["causal"])
        return (out, lse) if case["lse"] else out
    # rounded to the input's type between the operators, as the definition has it
    q, k = (_exact_rotate(s, x, 1.0).to(x.dtype).double() for x in (s.q, s.k))
    _exact_write(s, codes, scales, k, s.v.double())
    return [_exact_attend(s, codes, scales, q, True)[0], codes, scales]


def _exact_rotate(s, x, sign):
    y = x.double().clone()
    for i in range(s.axis.numel()):
        a, b = (2 * i, 2 * i + 1) if s.case["neighbours"] else (i, i + s.axis.numel())
        angle = s.positions[int(s.axis[i])].double() * s.frequency[i] * sign
        u, w = x[:, :, a].double(), x[:, :, b].double()
        y[:, :, a] = u * torch.cos(angle)[:, None] - w * torch.sin(angle)[:, None]
        y[:, :, b] = u * torch.sin(angle)[:, None] + w * torch.cos(angle)[:, None]
    return y


def _two_to(e):
    """2^e in 64 bits, from numbers that are exact (the GPU's pow is not)."""
    return torch.tensor([2.0 ** i for i in range(-300, 301)], dtype=torch.float64, device="cuda")[e.long() + 300]


def _nearest_e4m3(x):
    """Ties to even; subnormal numbers share the smallest binade's spacing 2^-9."""
    step = _two_to(torch.frexp(x.abs().clamp(min=2.0 ** -6))[1] - 4)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_write(s, codes, scales, k, v):
    fmt, T = s.case["format"], s.case["page"]
    nearest = _nearest_e4m3 if fmt == E4M3 else lambda x: torch.round(x).clamp(-127, 127)
    powers = _two_to(torch.arange(LOWEST, HIGHEST[fmt] + 1, device="cuda"))
    starts, table = s.row_starts.tolist(), s.table.tolist()
    for b, (n, r) in enumerate(zip(s.held, s.rows)):
        for first in range(n // T * T, n + r, T):
            page = table[b][first // T]
            t0, t1 = max(first, n) - first, min(first + T, n + r) - first
            x = torch.stack([z[starts[b] + first + t0 - n:starts[b] + first + t1 - n] for z in (k, v)]).permute(2, 0, 1, 3)
            largest = x.abs().amax((2, 3)).unsqueeze(-1)                                     # [heads][K|V][1]
            scale = powers[((largest > powers * LARGEST[fmt]).sum(-1)).clamp(max=len(powers) - 1)]
            if t0:
                scale = torch.maximum(scale, scales[page])
                codes[page, :, :, :t0] = nearest(codes[page, :, :, :t0] * (scales[page] / scale)[..., None, None])
            codes[page, :, :, t0:t1] = nearest(x / scale[..., None, None])
            scales[page] = scale


def _exact_read(s, scales):
    T, table, k, v = s.case["page"], s.table.tolist(), [], []
    for b, (n, r) in enumerate(zip(s.held, s.rows)):
        pages = torch.tensor(table[b], device="cuda")
        for rows, which in ((k, 0), (v, 1)):
            x = s.codes[pages, :, which].double() * scales[pages, :, which, None, None]
            rows.append(x.transpose(1, 2).flatten(0, 1)[n:n + r])
    return [torch.cat(k), torch.cat(v)]


def _exact_attend(s, codes, scales, q, causal):
    H, d, group = s.case["kv_heads"], s.case["dim"], s.case["q_heads"] // s.case["kv_heads"]
    out, lse, at = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda"), 0
    for b, (n, r) in enumerate(zip(s.held, s.rows)):
        n = n + r
        pages = s.table[b].long()
        hidden = torch.arange(n, device="cuda") > torch.arange(r, device="cuda")[:, None] + (n - r if causal else n)
        for h in range(H):
            k, v = ((codes[pages, h, w].double() * scales[pages, h, w, None, None]).flatten(0, 1)[:n] for w in (0, 1))
            mine = slice(h * group, (h + 1) * group)
            z = torch.einsum("rgd,nd->grn", q[at:at + r, mine], k) / d ** 0.5
            z = torch.where(hidden, -math.inf, z)
            lse[at:at + r, mine] = torch.logsumexp(z, -1).T
            out[at:at + r, mine] = (torch.softmax(z, -1) @ v).transpose(0, 1)
        at += r
    return out, lse
