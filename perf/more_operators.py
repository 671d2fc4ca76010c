"""Decode steps over the paged cache of bf16 or fp32 rows, as cases that a timing or comparison harness can run.

Kinds of case
  append  rotary positions of new queries and keys, and the keys and values into their slots of the cache's pages
          (`append_paged`); with `bounds` also each page's lowest and largest key of every column.
  bounds  those bounds of all pages that hold rows (`page_bounds`).
  shared  one decode step of sequences that share the rows of a prompt and have rows of their own
          (`decode_attention_shared`).
  chosen  for each sequence, layer and KV head the pages with the largest possible scores, and a decode step of attention
          over these pages alone (`choose_pages`, `decode_attention_chosen`).

`run` computes them in plain torch operations where `own` is false, and through the package where it is true.
`exact` has the same in 64 bits, from the definitions.

A page's score for the G query heads of a KV head is the sum over them of the largest dot product that a key within the
page's bounds can have, sum_g sum_c max(q_gc low_c, q_gc high_c), in 64 bits, rounded to 32.  The `first` and the `last`
pages of a unit are taken whatever their scores, then those of largest score, the earlier one of two alike, until there
are `count`; pages that the block table lacks are left out.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ----------------------------------------------------------------------------------
def _case(name, kind, **over):
    c = {"name": name, "kind": kind, "dtype": "bf16", "batch": 1, "layers": 28, "kv_heads": 4, "group": 7, "head_dim": 128, "page": 64}
    c.update({
        "append": {"layers": 1, "tokens": 1, "held": 0, "rotary_dim": 128, "interleaved": False, "scaling": "none", "factor": 1.0,
                   "streams": 1, "bounds": False},
        "bounds": {"tokens": 32768, "rho": 0.2, "holes": False},
        "shared": {"tokens": 32768, "rho": 0.2, "prefixes": 1, "loose": 0, "rows": 256, "holes": False},
        "chosen": {"tokens": 32768, "rho": 1.0, "count": 64, "first": 1, "last": 2, "holes": False}}[kind])
    return {**c, **over}


def listed():
    return [
        # the smallest step: one fp32 layer of a short context
        _case("append_tiny", "append", dtype="f32", kv_heads=2, group=4, head_dim=64, rotary_dim=64, held=102, page=16),
        # a decode step of one layer, eight sequences, multimodal positions in three streams, pages ranked by their bounds
        _case("append_step", "append", batch=8, held=1638, streams=3, bounds=True),
        # a chunk of two prompts behind what they hold already, interleaved pairs of half of the columns
        _case("append_chunk", "append", batch=2, tokens=1003, held=2021, kv_heads=8, group=4, rotary_dim=64, interleaved=True, page=48, bounds=True),
        # one layer of a long prompt into an empty cache, context extended by parts
        _case("append_prompt", "append", tokens=32768, scaling="parts", factor=4.0),
        # the bounds of one layer's pages for eight compressed prompts
        _case("bounds_layer", "bounds", batch=8, layers=1, tokens=16384, rho=0.1, page=32),
        # the bounds of all pages of a long prompt's compressed cache, once after the prompt
        _case("bounds_32k", "bounds"),
        # eight answers to one compressed prompt, one layer's decode step as a model runs it
        _case("shared_layer", "shared", batch=8, layers=1),
        # sixteen answers to one compressed prompt, all layers' rows
        _case("shared_32k", "shared", batch=16),
        # a server's batch: four prompts with different numbers of answers, two sequences without a shared prompt, an fp32 cache
        _case("shared_mixed", "shared", dtype="f32", batch=27, layers=4, tokens=8192, rho=0.3, prefixes=4, loose=2, group=4, rows=700, page=32),
        # one layer's decode step over the best pages of a long prompt that was not compressed
        _case("chosen_layer", "chosen", layers=1, count=32),
        # all layers of that prompt
        _case("chosen_32k", "chosen"),
        # eight compressed sequences in small pages, of which a quarter is read
        _case("chosen_batch8", "chosen", batch=8, tokens=16384, rho=0.1, page=16, count=26, holes=True),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(["append", "append", "bounds", "shared", "shared", "chosen", "chosen"])
    case = _case("", kind, dtype="f32" if rng.random() < 0.25 else "bf16", kv_heads=rng.choice([1, 2, 4, 8]),
                 group=rng.choice([1, 2, 3, 4, 7, 8, 16]), head_dim=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 48, 64, 128]))
    e = 2 if case["dtype"] == "f32" else 1
    if kind == "append":
        d = case["head_dim"] = rng.choice([64, 128, 128, 80])
        case.update(batch=rng.choice([1, 1, 2, 8, 32]), tokens=int(_log_uniform(rng, 1, 33000)), held=rng.choice([0, int(_log_uniform(rng, 1, 5000))]),
                    rotary_dim=rng.choice([d, d, d // 2]), interleaved=rng.random() < 0.4, scaling=rng.choice(["none", "linear", "base", "parts"]),
                    factor=rng.choice([2.0, 4.0, 8.0]), streams=rng.choice([1, 1, 3]), bounds=rng.random() < 0.5)
        if rng.random() < 0.4:
            case["tokens"] = 1
        # no more than the largest listed case: its columns of queries, keys and values, and as much cache
        while case["batch"] * case["kv_heads"] * d * e * max(case["tokens"] * (case["group"] + 2), (case["tokens"] + case["held"]) * 4) > 32768 * 36 * 128:
            if case["batch"] > 1:
                case["batch"] //= 2
            else:
                case["tokens"], case["held"] = max(1, case["tokens"] * 3 // 4), case["held"] * 3 // 4
        del case["name"]
        return case
    case.update(batch=rng.choice([1, 1, 2, 3, 8]), layers=int(round(_log_uniform(rng, 1, 36))), tokens=int(_log_uniform(rng, 100, 66000)),
                rho=round(_log_uniform(rng, 0.05, 1.0), 4), holes=rng.random() < 0.3)
    if kind == "shared":
        case.update(batch=int(round(_log_uniform(rng, 1, 40))), rows=rng.choice([0, int(_log_uniform(rng, 1, 3000))]))
        case["prefixes"] = rng.randint(1, min(5, case["batch"]))
        case["loose"] = rng.choice([0, 0, 1, 3]) if case["batch"] > case["prefixes"] + 3 else 0
    elif kind == "chosen":
        case.update(count=int(_log_uniform(rng, 1, 200)), first=rng.choice([0, 1, 2]), last=rng.choice([0, 1, 2, 4]))
        case["count"] = max(case["count"], case["first"] + case["last"])
    # no more than the largest listed case of the kind
    whole = {"bounds": 28 * 4 * 6554 * 128, "shared": 28 * 4 * (6554 + 16 * 128) * 128, "chosen": 28 * 4 * 32768 * 128}[kind]
    least = 28 * 4 * 64 * 64 * 128
    while True:
        units = case["layers"] * case["kv_heads"] * case["head_dim"] * e
        held = case["tokens"] * case["rho"]
        if kind == "shared":
            rows = units * (case["prefixes"] * held + case["batch"] * case["rows"] / 2)
            pairs = units * case["batch"] * case["group"] * (held + case["rows"] / 2)
            if rows <= whole and pairs <= 28 * 4 * 128 * 16 * 7 * 6700:
                break
        elif kind == "bounds":
            if units * case["batch"] * held <= whole:
                break
        elif units * case["batch"] * held <= whole and units * case["batch"] * min(held, case["count"] * case["page"]) <= least:
            break
        if kind != "shared" and case["batch"] > 1:
            case["batch"] = 1
        elif case["layers"] > 4:
            case["layers"] //= 2
        elif case["tokens"] > 200:
            case["tokens"], case["rows"] = case["tokens"] * 3 // 4, case.get("rows", 0) * 3 // 4
        else:
            case["kv_heads"] = max(1, case["kv_heads"] // 2)
            case["group"] = max(1, case["group"] // 2)
    if kind != "shared":
        case.pop("rows", None)
    del case["name"]
    return case


# ---- inputs ---------------------------------------------------------------------------------
def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _kept(batch, case, gen):
    """Rows [batch, L] that the layers keep, the same in all for each sequence: shares that differ as the allocation makes them differ."""
    L, N, rho = case["layers"], case["tokens"], case["rho"]
    total = max(L, int(rho * L * N))
    spread = min(1.0, 1.98 * (1.0 - rho) / (1.0 + rho))                # (no share above N)
    w = 1.0 + spread * (torch.rand((batch, L), generator=gen, device="cuda", dtype=torch.float64) - 0.5)
    rows = ((total - L) * w / w.sum(1, keepdim=True)).floor().to(torch.int64) + 1
    left = total - rows.sum(1, keepdim=True)                           # fewer than L: a row each to the first layers
    return rows + (torch.arange(L, device="cuda") < left)


def _values(shape, gen, dtype):
    """Rows around a mean for each column, some columns far larger than the others, as keys have them."""
    x = torch.randn(shape, generator=gen, device="cuda")
    wide = 1.0 + 4.0 * (torch.rand((shape[-1],), generator=gen, device="cuda") > 0.94).float()
    return (x * wide + 0.5 * torch.randn((shape[-1],), generator=gen, device="cuda")).to(dtype)


def _cache(rows, heads, case, gen, most_rows):
    """A cache whose units (sequence, layer, head) hold rows [B, L], in pages at random places: the pages' K and V, the table."""
    B, L = rows.shape
    ps, d, dt = case["page"], case["head_dim"], _DTYPES[case["dtype"]]
    most = max(1, -(-most_rows // ps))
    need = (-(-rows // ps)).repeat_interleave(heads, 1).reshape(-1)
    total = int(need.sum())
    free = torch.randperm(total + 3, generator=gen, device="cuda").to(torch.int32)
    at = torch.arange(most, device="cuda")
    first = torch.cumsum(need, 0) - need
    table = torch.where(at < need[:, None], free[(first[:, None] + at).clamp(max=total + 2)], -1).view(B, L, heads, most)
    if case.get("holes"):                                              # layers without rows, and pages that are gone
        rows = torch.where(torch.rand((B, L), generator=gen, device="cuda") < 0.15, 0, rows)
        table = torch.where(torch.rand(table.shape, generator=gen, device="cuda") < 0.1, -1, table)
    shape = (total + 3, ps, d)
    # keys that follow each other are alike: a page's rows lie around a point of its own
    K = (_values((total + 3, 1, d), gen, torch.float32) + 0.5 * torch.randn(shape, generator=gen, device="cuda")).to(dt)
    return {"K": K, "V": _values(shape, gen, dt), "table": table.contiguous(), "rows": rows.to(torch.int32)}


def _frequencies(case):
    R, s = case["rotary_dim"], case["factor"]
    theta = 1.0e6
    if case["scaling"] == "base":
        theta *= s ** (R / max(1, R - 2))
    f = [theta ** (-2.0 * i / R) for i in range(R // 2)]
    if case["scaling"] == "linear":
        return [x / s for x in f], 1.0
    if case["scaling"] == "parts":
        ramp = [min(1.0, max(0.0, (32768 * x / (2.0 * math.pi) - 1.0) / 31.0)) for x in f]
        return [x * g + x / s * (1.0 - g) for x, g in zip(f, ramp)], 0.1 * math.log(s) + 1.0
    return f, 1.0


def _sections(case):
    """Pairs that each stream of positions turns."""
    half = case["rotary_dim"] // 2
    if case["streams"] == 1:
        return (half,)
    third = half * 3 // 8
    return (half - 2 * third, third, third)


def _starts(case):
    """First sequence of each prompt's, and the end of the last one's: 1, 2, 3, ... parts, half of those without a prompt in front."""
    P, B = case["prefixes"], case["batch"] - case["loose"]
    parts = P * (P + 1) // 2
    return [case["loose"] // 2 + (B - P) * (p * (p + 1) // 2) // parts + p for p in range(P + 1)]


def _page_bounds(K, rows, table):
    """Lowest and largest key [num_pages, 2, d] of the pages that hold rows; zeros elsewhere."""
    B, L, H, most = table.shape
    ps = K.shape[1]
    out = torch.zeros((K.shape[0], 2, K.shape[2]), dtype=K.dtype, device="cuda")
    in_page = (rows.long()[:, :, None, None] - ps * torch.arange(most, device="cuda")).clamp(0, ps).expand(B, L, H, most)
    some = (in_page > 0) & (table >= 0)
    page, n = table[some].long(), in_page[some]
    for a in range(0, page.numel(), 8192):
        x, dead = K[page[a:a + 8192]], (torch.arange(ps, device="cuda") >= n[a:a + 8192, None])[:, :, None]
        out[page[a:a + 8192], 0] = x.masked_fill(dead, math.inf).amin(1)
        out[page[a:a + 8192], 1] = x.masked_fill(dead, -math.inf).amax(1)
    return out


def _prepare_append(case, gen, s):
    dt = _DTYPES[case["dtype"]]
    B, T, H, G, d, ps, held = (case[k] for k in ("batch", "tokens", "kv_heads", "group", "head_dim", "page", "held"))
    c = _cache(torch.full((B, 1), held + T, dtype=torch.int64, device="cuda"), H, case, gen, held + T)
    # queries, keys and values as one projection leaves them
    x = torch.randn((B, T, (G + 2) * H, d), generator=gen, device="cuda").to(dt)
    s["Q"], s["new_K"], s["new_V"] = x[:, :, :G * H], x[:, :, G * H:(G + 1) * H], x[:, :, (G + 1) * H:]
    first = torch.randint(0, 100000, (case["streams"], B, 1), generator=gen, device="cuda")
    s["positions"] = (first + torch.arange(T, device="cuda") // (1 + torch.arange(case["streams"], device="cuda"))[:, None, None]).to(torch.int32)
    f, magnitude = _frequencies(case)
    s["magnitude"] = magnitude
    s["frequencies"] = torch.tensor(f, dtype=torch.float64, device="cuda")
    s["stream"] = torch.repeat_interleave(torch.arange(case["streams"], device="cuda"), torch.tensor(_sections(case), device="cuda"))
    # slots of two layers in the order of layer, head, row, of which this is the second
    row = held + torch.arange(T, device="cuda")
    slots = c["table"].long()[:, 0].gather(2, (row // ps).expand(B, H, T)) * ps + row % ps
    s["slots"] = torch.cat((torch.full_like(slots, -1), slots), 1)[:, H:]
    s["K"], s["V"] = c["K"], c["V"]
    s["bounds"] = _page_bounds(c["K"], torch.full((B, 1), held, device="cuda"), c["table"]) if case["bounds"] else None
    s["Q_out"] = torch.empty((B, T, G * H, d), dtype=dt, device="cuda")
    if own:
        s["plan"] = s["fc"].rotary_plan(case["rotary_dim"], theta=1.0e6, interleaved=case["interleaved"], scaling=case["scaling"],
                                        factor=case["factor"], original_tokens=32768, sections=_sections(case) if case["streams"] > 1 else None)


def prepare(case, seed):
    gen = _generator(seed)
    kind = case["kind"]
    s = {"case": case}
    if own:
        import paper_2511_16786_amd as fc
        s["fc"] = fc
    if kind == "append":
        _prepare_append(case, gen, s)
        return s
    B, L, H, G, d = (case[k] for k in ("batch", "layers", "kv_heads", "group", "head_dim"))
    dt = _DTYPES[case["dtype"]]
    s["cache"] = _cache(_kept(case["prefixes"] if kind == "shared" else B, case, gen), H, case, gen, case["tokens"])
    if kind != "shared":
        c = s["cache"]
        s["bounds"] = _page_bounds(c["K"], c["rows"], c["table"]) if kind == "chosen" else torch.zeros((c["K"].shape[0], 2, d), dtype=dt, device="cuda")
    if kind != "bounds":
        s["Q"] = torch.randn((B, L, H * G, d), generator=gen, device="cuda").to(dt)
        s["out"] = torch.empty((B, L, H * G, d), dtype=torch.float32, device="cuda")
    if kind == "shared":
        # sequences that began one after another, the last one just now
        rows = torch.tensor([case["rows"] * b // max(1, B - 1) for b in range(B)], device="cuda")
        s["mine"] = _cache(rows[:, None].expand(B, L), H, case, gen, case["rows"] + 1)
        s["starts"] = torch.tensor(_starts(case), dtype=torch.int32, device="cuda")
    if kind == "chosen":
        s["chosen"] = torch.empty((B, L, H, case["count"]), dtype=torch.int32, device="cuda")
    if own:
        fc = s["fc"]
        s["paged"] = fc.PagedKV(*(s["cache"][k] for k in ("K", "V", "rows", "table")))
        if kind == "shared":
            s["paged_mine"] = fc.PagedKV(*(s["mine"][k] for k in ("K", "V", "rows", "table")))
            s["workspace"] = fc.shared_workspace(s["Q"], H, case["prefixes"])
        elif kind == "chosen":
            s["workspace"] = fc.chosen_workspace(s["Q"], s["paged"], case["count"])
    return s


# ---- plain forms ----------------------------------------------------------------------------
def _turn(x, cos, sin, R, interleaved):
    out = x.float()
    a, b = (out[..., 0:R:2], out[..., 1:R:2]) if interleaved else (out[..., :R // 2], out[..., R // 2:R])
    p, q = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((p, q), -1).flatten(-2) if interleaved else torch.cat((p, q), -1)
    return torch.cat((turned, out[..., R:]), -1).to(x.dtype)


def _plain_append(s):
    case = s["case"]
    d, ps, R = case["head_dim"], case["page"], case["rotary_dim"]
    angle = s["positions"].double()[s["stream"]].permute(1, 2, 0) * s["frequencies"]
    cos = (angle.cos() * s["magnitude"]).float()[:, :, None]
    sin = (angle.sin() * s["magnitude"]).float()[:, :, None]
    Q, K = (_turn(s[n], cos, sin, R, case["interleaved"]) for n in ("Q", "new_K"))
    slots = s["slots"].transpose(1, 2)                                 # [B, T, H], as the rows are
    s["K"].view(-1, d)[slots] = K
    s["V"].view(-1, d)[slots] = s["new_V"]
    out = {"Q": Q, "K": s["K"], "V": s["V"]}
    if case["bounds"]:
        page, at = slots // ps, slots % ps
        begun = page[at == 0]
        s["bounds"][begun, 0], s["bounds"][begun, 1] = math.inf, -math.inf
        place = page.reshape(-1, 1).expand(-1, d)
        s["bounds"][:, 0] = s["bounds"][:, 0].scatter_reduce(0, place, K.reshape(-1, d), "amin")
        s["bounds"][:, 1] = s["bounds"][:, 1].scatter_reduce(0, place, K.reshape(-1, d), "amax")
        out["bounds"] = s["bounds"]
    return out


def _plain_bounds(s):
    c = s["cache"]
    return _page_bounds(c["K"], c["rows"], c["table"])


def _gathered(c, j, units):
    """fp32 rows j of some units' pages (table entries [n, pages], row counts [n]), and which of them there are."""
    table, rows = units
    ps, d = c["K"].shape[1:]
    most = table.shape[1]
    page = table.long()[:, (j // ps).clamp(max=most - 1)]
    ok = (j < rows[:, None]) & (j < most * ps) & (page >= 0) & (page < c["K"].shape[0])
    slot = torch.where(ok, page * ps + j % ps, 0)
    return c["K"].view(-1, d)[slot].float(), c["V"].view(-1, d)[slot].float(), ok


def _logits(q, K, ok):
    return (torch.matmul(q, K.transpose(1, 2).contiguous()) / math.sqrt(q.shape[-1])).masked_fill(~ok[:, None], -math.inf)


def _units(c, which):
    """Tables [n, pages] and row counts [n] of the units of the sequences `which`."""
    table, rows = c["table"][which], c["rows"][which]
    H = table.shape[2]
    return table.flatten(0, 2), rows.flatten().repeat_interleave(H)


def _plain_shared(s):
    case = s["case"]
    B, L, Hq, d = s["Q"].shape
    H, G = case["kv_heads"], case["group"]
    starts = _starts(case)
    parts = [(p, starts[p], starts[p + 1]) for p in range(case["prefixes"])]
    parts += [(None, a, b) for a, b in ((0, starts[0]), (starts[-1], B)) if b > a]
    out = torch.empty((B, L, H, G, d), device="cuda")
    j_mine = torch.arange(max(1, int(case["rows"])), device="cuda")
    j_all = torch.arange(max(1, int(s["cache"]["rows"].max())), device="cuda")
    for p, a, b in parts:
        m = b - a
        q = s["Q"][a:b].float().view(m, L, H, G, d)
        K, V, ok = _gathered(s["mine"], j_mine, _units(s["mine"], slice(a, b)))
        mine, q_mine = V, q.reshape(m * L * H, G, d)
        logit = _logits(q_mine, K, ok).view(m, L, H, G, -1)
        top = logit.amax(4, keepdim=True)
        if p is not None:
            K, V, ok = _gathered(s["cache"], j_all, _units(s["cache"], slice(p, p + 1)))
            q_all = q.permute(1, 2, 0, 3, 4).reshape(L * H, m * G, d)
            common = _logits(q_all, K, ok).view(L, H, m, G, -1).permute(2, 0, 1, 3, 4)
            top = torch.maximum(top, common.amax(4, keepdim=True))
        top = torch.where(top == -math.inf, 0.0, top)
        w = torch.exp(logit - top)
        total = w.sum(4, keepdim=True)
        acc = torch.matmul(w.view(m * L * H, G, -1), mine).view(m, L, H, G, d)
        if p is not None:
            w = torch.exp(common - top)
            total = total + w.sum(4, keepdim=True)
            acc = acc + torch.matmul(w.permute(1, 2, 0, 3, 4).reshape(L * H, m * G, -1), V).view(L, H, m, G, d).permute(2, 0, 1, 3, 4)
        out[a:b] = acc / torch.where(total == 0.0, 1.0, total)
    return out.view(B, L, Hq, d)


def _plain_chosen(s):
    case, c = s["case"], s["cache"]
    B, L, H, most = c["table"].shape
    G, d, ps, count = case["group"], case["head_dim"], case["page"], case["count"]
    q = s["Q"].view(B, L, H, G, d)
    wide = q.double()
    table, blocks = c["table"].long(), ((c["rows"].long() + ps - 1) // ps)[:, :, None, None]
    at = torch.arange(most, device="cuda")
    there = (at < blocks) & (table >= 0)
    taken = torch.where(there, table, 0)
    score = torch.empty((B, L, H, most), device="cuda")
    for b in range(B):                                                 # (a sequence at a time: 64-bit bounds of all would not be small)
        low, high = s["bounds"][taken[b]].double().unbind(3)
        up, down = wide[b].clamp(min=0.0).sum(2), wide[b].clamp(max=0.0).sum(2)
        score[b] = ((high * up[:, :, None]).sum(3) + (low * down[:, :, None]).sum(3)).float()
    forced = (at < case["first"]) | (at >= blocks - case["last"])
    score = torch.where(there, torch.where(forced, math.inf, score), -math.inf)
    order = torch.sort(score, dim=3, descending=True, stable=True).indices[..., :count]
    found = torch.gather(there, 3, order)
    order = torch.where(found, order, most).sort(3).values
    if order.shape[3] < count:
        order = torch.cat((order, torch.full((B, L, H, count - order.shape[3]), most, device="cuda")), 3)
    chosen = torch.where(order < most, order, -1).to(torch.int32)
    out = torch.empty((B, L, H, G, d), device="cuda")
    n = chosen.clamp(min=0).long()
    row = (n[..., None] * ps + torch.arange(ps, device="cuda")).flatten(3)
    ok = (chosen >= 0).repeat_interleave(ps, 3) & (row < c["rows"].long()[:, :, None, None])
    slot = torch.where(ok, ((taken.gather(3, n) * ps)[..., None] + torch.arange(ps, device="cuda")).flatten(3), 0)
    for b in range(B):
        K, V = (c[x].view(-1, d)[slot[b].flatten(0, 1)].float() for x in ("K", "V"))
        logit = _logits(q[b].float().flatten(0, 1), K, ok[b].flatten(0, 1))
        top = logit.amax(2, keepdim=True)
        w = torch.exp(logit - torch.where(top == -math.inf, 0.0, top))
        total = w.sum(2, keepdim=True)
        out[b] = (torch.matmul(w, V) / torch.where(total == 0.0, 1.0, total)).view(L, H, G, d)
    return {"chosen": chosen, "out": out.view(B, L, H * G, d)}


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        return {"append": _plain_append, "bounds": _plain_bounds, "shared": _plain_shared, "chosen": _plain_chosen}[kind](s)
    fc = s["fc"]
    if kind == "append":
        fc.append_paged(s["plan"], s["positions"], s["Q"], s["new_K"], s["new_V"], s["slots"], s["K"], s["V"], Q_out=s["Q_out"], bounds=s["bounds"])
        out = {"Q": s["Q_out"], "K": s["K"], "V": s["V"]}
        if case["bounds"]:
            out["bounds"] = s["bounds"]
        return out
    if kind == "bounds":
        return fc.page_bounds(s["paged"], s["bounds"])
    scale = 1.0 / math.sqrt(case["head_dim"])
    if kind == "shared":
        return fc.decode_attention_shared(s["Q"], s["paged"], s["starts"], s["paged_mine"], scale, out=s["out"], workspace=s["workspace"])
    chosen = fc.choose_pages(s["Q"], s["paged"], s["bounds"], case["count"], first=case["first"], last=case["last"], chosen=s["chosen"],
                             workspace=s["workspace"])
    out = fc.decode_attention_chosen(s["Q"], s["paged"], chosen, scale, out=s["out"], workspace=s["workspace"])
    return {"chosen": chosen, "out": out}


# ---- 64 bits, from the definitions ----------------------------------------------------------
def _rows_of(c, b, l, h):
    """Slots of the rows of one unit that are there, and the rows' numbers."""
    ps = c["K"].shape[1]
    j = torch.arange(min(int(c["rows"][b, l]), ps * c["table"].shape[3]), device="cuda")
    page = c["table"][b, l, h].long()[j // ps]
    fine = page >= 0
    return (page * ps + j % ps)[fine], j[fine]


def _attended(q, K, V):
    """Softmax-weighted rows in 64 bits: q [n, d], K and V [rows, d]."""
    if not K.shape[0]:
        return torch.zeros_like(q)
    return torch.mm(torch.softmax(torch.mm(q, K.t()) / math.sqrt(q.shape[1]), 1), V)


def _exact_append(s, case):
    R, d, ps = case["rotary_dim"], case["head_dim"], case["page"]
    angle = s["positions"].double()[s["stream"]].movedim(0, -1) * s["frequencies"]
    turn = torch.polar(torch.full_like(angle, s["magnitude"]), angle)[:, :, None]

    def turned(x):
        x = x.double()
        pairs = x[..., :R].unflatten(-1, (R // 2, 2)) if case["interleaved"] else x[..., :R].unflatten(-1, (2, R // 2)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        z = z if case["interleaved"] else z.transpose(-1, -2)
        return torch.cat((z.reshape(*x.shape[:-1], R), x[..., R:]), -1)

    K, V, new = s["K"].double(), s["V"].double(), turned(s["new_K"])
    slots = s["slots"].transpose(1, 2).reshape(-1)
    K.view(-1, d)[slots] = new.reshape(-1, d)
    V.view(-1, d)[slots] = s["new_V"].double().reshape(-1, d)
    out = {"Q": turned(s["Q"]), "K": K, "V": V}
    if case["bounds"]:
        low_high = s["bounds"].double()
        touched = torch.zeros(K.shape[:2], dtype=torch.bool, device="cuda").view(-1)
        touched[slots] = True
        touched = touched.view(-1, ps)
        for lowest, sign in ((0, 1.0), (1, -1.0)):                     # the largest is the lowest of the negatives
            most = torch.where(touched[:, :, None], sign * K, math.inf).amin(1)
            before = torch.where(touched[:, :1], math.inf, sign * low_high[:, lowest])
            low_high[:, lowest] = sign * torch.where(touched.any(1)[:, None], torch.minimum(most, before), sign * low_high[:, lowest])
        out["bounds"] = low_high
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "append":
        return _exact_append(s, case)
    c = s["cache"]
    d, ps, H, G, L = (case[k] for k in ("head_dim", "page", "kv_heads", "group", "layers"))
    if kind == "bounds":
        out = torch.zeros((c["K"].shape[0], 2, d), dtype=torch.float64, device="cuda")
        for l in range(L):
            for b in range(case["batch"]):
                for h in range(H):
                    slot, j = _rows_of(c, b, l, h)
                    if not slot.numel():
                        continue
                    lists = torch.full((-(-int(c["rows"][b, l]) // ps), ps, d), math.nan, dtype=torch.float64, device="cuda")
                    lists.view(-1, d)[j] = c["K"].view(-1, d)[slot].double()
                    full = (~lists[:, 0, 0].isnan()).nonzero()[:, 0]
                    page = c["table"][b, l, h].long()[full]
                    out[page, 0] = lists[full].nan_to_num(nan=math.inf).min(1).values
                    out[page, 1] = lists[full].nan_to_num(nan=-math.inf).max(1).values
        return out
    Q = s["Q"].double()
    out = torch.zeros_like(Q)
    starts = _starts(case) if kind == "shared" else None
    for b in range(case["batch"]):
        for l in range(L):
            for h in range(H):
                q = Q[b, l, h * G:(h + 1) * G]
                if kind == "shared":
                    part = s["mine"]
                    slots = [_rows_of(part, b, l, h)[0]]
                    K, V = ([part[x].view(-1, d)[slots[0]].double()] for x in ("K", "V"))
                    for p in range(case["prefixes"]):
                        if starts[p] <= b < starts[p + 1]:
                            slot = _rows_of(c, p, l, h)[0]
                            K.append(c["K"].view(-1, d)[slot].double())
                            V.append(c["V"].view(-1, d)[slot].double())
                    out[b, l, h * G:(h + 1) * G] = _attended(q, torch.cat(K), torch.cat(V))
                    continue
                blocks = -(-int(c["rows"][b, l]) // ps)
                table = c["table"][b, l, h].long()[:blocks]
                there = (table >= 0).nonzero()[:, 0]
                if not there.numel():
                    continue
                low_high = s["bounds"][table[there]].double()
                best = torch.maximum(q[:, None] * low_high[:, 0], q[:, None] * low_high[:, 1]).sum((0, 2)).float()
                kept = (there < case["first"]) | (there >= blocks - case["last"])
                left = min(case["count"], there.numel()) - int(kept.sum())
                if left > 0:
                    rank = torch.argsort(torch.where(kept, -math.inf, best), descending=True, stable=True)[:left]
                    kept[rank] = True
                elif left < 0:
                    raise ValueError("more pages are taken whatever their scores than may be chosen")
                slot, j = _rows_of(c, b, l, h)
                mine = torch.isin(j // ps, there[kept])
                out[b, l, h * G:(h + 1) * G] = _attended(q, *(c[x].view(-1, d)[slot[mine]].double() for x in ("K", "V")))
    return out if kind == "shared" else {"chosen": None, "out": out}


def work(case):
    """Every input read once and every output written once."""
    e = 2 if case["dtype"] == "bf16" else 4
    B, L, H, G, d, ps = (case[k] for k in ("batch", "layers", "kv_heads", "group", "head_dim", "page"))
    if case["kind"] == "append":
        rows = B * case["tokens"] * H
        moved = 2 * rows * (G + 2) * d * e + 8 * rows + 4 * case["streams"] * B * case["tokens"]
        if case["bounds"]:                                             # of the pages that rows go to
            moved += 2 * d * e * B * H * (2 if case["tokens"] == 1 else -(-case["tokens"] // ps))
        return {"bytes": moved, "flops": 3 * rows * (G + 1) * case["rotary_dim"]}
    kept = H * max(L, int(case["rho"] * L * case["tokens"]))            # rows of a sequence, or of a prompt
    pages = -(-kept // ps)
    if case["kind"] == "bounds":
        return {"bytes": B * (kept * d * e + pages * (2 * d * e + 4)), "flops": 2 * B * kept * d}
    q = B * L * H * G * d
    if case["kind"] == "shared":
        mine = L * H * sum(case["rows"] * b // max(1, B - 1) for b in range(B))
        return {"bytes": 2 * d * e * (case["prefixes"] * kept + mine) + q * (e + 4),
                "flops": 4 * G * d * ((B - case["loose"]) * kept + mine)}
    read = min(kept, L * H * case["count"] * ps)
    return {"bytes": B * (pages * (2 * d * e + 4) + 2 * read * d * e + 4 * L * H * case["count"]) + q * (e + 4),
            "flops": B * (4 * pages * d + 4 * G * d * read)}
