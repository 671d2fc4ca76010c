"""The decode loop's operators around a compacted cache, as cases that a timing or comparison harness can run.

Kinds of case
  rotary  rotary positions of the queries and keys of new tokens (`rotary`).
  pages   block tables and slot maps from the rows that sequences hold and add (`assign_pages`).
  store   rows into the 4-bit paged cache and back (`mx_store`, `mx_load`).
  gather  selection from given scores straight into the 4-bit paged cache, and the rows read back
          (`select_gather_mx`, `mx_load`).
  attend  one decode step of attention over the 4-bit paged cache (`mx_decode_attention`).

`run` computes them in plain torch operations where `own` is false, and through the package where it is true.
`exact` has the same in 64 bits, from the definitions.

The 4-bit format.  32 neighbouring columns share a power of two 2^(E - 127), E = ((bits(m) + 2^21) >> 23) - 2 clamped to
[2, 252] with m the largest magnitude as fp32 (so that m / 2^(E - 127) is below 7); a value is one sign and three bits
e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6), rounded to nearest, ties to the even code, saturating.  Sixteen slots of K and V of d
columns are a tile of 17 d bytes: K codes [16][d/2], V codes [4][16][4][d/32] (row quad, d/16 columns, row of the quad), K
scales [d/32][16], V scales [4][d/32][4] (row quad, block, row of the quad); the lower nibble is the even column.
"""
import functools
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ----------------------------------------------------------------------------------
def _rotary(name, **over):
    c = {"name": name, "kind": "rotary", "dtype": "bf16", "batch": 1, "tokens": 1, "q_heads": 28, "kv_heads": 4,
         "head_dim": 128, "rotary_dim": 128, "interleaved": False, "scaling": "none", "factor": 1.0, "streams": 1,
         "inverse": False, "far": 32768}
    return {**c, **over}


def _cached(name, kind, **over):
    c = {"name": name, "kind": kind, "dtype": "bf16", "batch": 1, "layers": 28, "kv_heads": 4, "head_dim": 128,
         "tokens": 32768, "rho": 0.2, "page": 64}
    c.update({"pages": {"add": 0}, "store": {"step": False}, "gather": {"shared": False},
              "attend": {"group": 7, "holes": False}}[kind])
    return {**c, **over}


def listed():
    return [
        # a decode step's queries and keys of one layer, multimodal positions in three streams
        _rotary("rotary_step", batch=8, streams=3),
        # a long prompt's queries and keys of one layer, context extended by parts
        _rotary("rotary_prompt", tokens=32768, scaling="parts", factor=4.0, far=131072),
        # tables and slots for the rows that a long prompt's compression keeps
        _cached("pages_prompt", "pages"),
        # a decode step of eight sequences: one row more for every unit
        _cached("pages_step", "pages", batch=8, tokens=16384, rho=0.1, add=1),
        # the new rows of a decode step of eight sequences, all layers
        _cached("store_step", "store", batch=8, tokens=16384, rho=0.1, step=True),
        # a compacted cache of a long prompt, packed rows as the selection left them
        _cached("store_32k", "store"),
        # a multi-image prompt compacted straight into four bits
        _cached("gather_8k", "gather", tokens=8192),
        # the long prompt, the headline workload's cache
        _cached("gather_32k", "gather"),
        # the smallest decode step: one fp32 layer of a short prompt
        _cached("attend_tiny", "attend", dtype="f32", layers=1, kv_heads=2, head_dim=64, tokens=512, group=4, page=16),
        # one layer's decode step as a model runs it, layer after layer
        _cached("attend_layer", "attend", layers=1),
        # all layers' rows of the long prompt
        _cached("attend_32k", "attend"),
        # eight sequences
        _cached("attend_batch8", "attend", batch=8, tokens=16384, rho=0.1, page=32),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(["rotary", "pages", "store", "gather", "attend", "attend"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if kind == "rotary":
        d = rng.choice([64, 128, 128, 80])
        case = _rotary("", dtype=dtype, batch=rng.choice([1, 1, 2, 8]), tokens=int(_log_uniform(rng, 1, 33000)),
                       q_heads=rng.choice([7, 16, 28, 32]), kv_heads=rng.choice([1, 4, 8]), head_dim=d,
                       rotary_dim=rng.choice([d, d, d // 2, d // 4 // 2 * 2]), interleaved=rng.random() < 0.4,
                       scaling=rng.choice(["none", "linear", "base", "parts"]), factor=rng.choice([2.0, 4.0, 8.0]),
                       streams=rng.choice([1, 1, 3]), inverse=rng.random() < 0.25, far=int(_log_uniform(rng, 1000, 2000000)))
        while case["batch"] * case["tokens"] * (case["q_heads"] + case["kv_heads"]) * d * (4 if dtype == "f32" else 2) > \
                32768 * 32 * 128 * 2:
            case["batch"], case["tokens"] = 1, max(1, case["tokens"] * 3 // 4)
    else:
        case = _cached("", kind, dtype=dtype, batch=rng.choice([1, 1, 2, 3, 8]), layers=int(round(_log_uniform(rng, 1, 36))),
                       kv_heads=rng.choice([1, 2, 4, 8]), head_dim=rng.choice([64, 128, 128]),
                       tokens=int(_log_uniform(rng, 100, 66000)), rho=round(_log_uniform(rng, 0.05, 0.95), 4),
                       page=rng.choice([16, 32, 48, 64, 128]))
        if kind == "pages":
            case["add"] = rng.choice([0, 0, 1, 3, 17])
        elif kind == "store":
            case["step"] = rng.random() < 0.4
        elif kind == "gather":
            case["shared"] = rng.random() < 0.3
        else:
            case["group"] = rng.choice([1, 2, 3, 4, 7, 8, 16])
            case["holes"] = rng.random() < 0.4
        # no more than the largest listed cases: their kept rows, and for a gather also the cache it selects from
        most, whole = {"pages": 28 * 4 * 6554, "store": 28 * 4 * 6554, "gather": 28 * 4 * 6554, "attend": 8 * 28 * 4 * 1638}[kind], 28 * 4 * 32768
        e = 2 if dtype == "f32" and kind != "attend" else 1
        while True:
            units = case["batch"] * case["layers"] * case["kv_heads"]
            if units * case["tokens"] * case["rho"] * e <= most and (kind != "gather" or units * case["tokens"] * e <= whole):
                break
            if case["batch"] > 1:
                case["batch"] = 1
            elif case["layers"] > 4:
                case["layers"] //= 2
            else:
                case["tokens"] = case["tokens"] * 3 // 4
    del case["name"]
    return case


# ---- inputs ---------------------------------------------------------------------------------
def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _rows(case, gen):
    """Rows [B, L] that the layers keep, of each sequence the same in all: shares that differ as the allocation makes them differ."""
    B, L, N, rho = case["batch"], case["layers"], case["tokens"], case["rho"]
    total = max(L, int(rho * L * N))
    spread = min(1.0, 1.98 * (1.0 - rho) / (1.0 + rho))                # (no share above N)
    w = 1.0 + spread * (torch.rand((B, L), generator=gen, device="cuda", dtype=torch.float64) - 0.5)
    rows = ((total - L) * w / w.sum(1, keepdim=True)).floor().to(torch.int64) + 1
    left = total - rows.sum(1, keepdim=True)                           # fewer than L: a row each to the first layers
    return rows + (torch.arange(L, device="cuda") < left)


def _values(shape, gen, dtype):
    """Rows around a slowly varying mean for each column, some columns far larger than the others, as keys have them."""
    x = torch.randn(shape, generator=gen, device="cuda")
    wide = 1.0 + 4.0 * (torch.rand((shape[-1],), generator=gen, device="cuda") > 0.94).float()
    return (x * wide + 0.5 * torch.randn((shape[-1],), generator=gen, device="cuda")).to(dtype)


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


def prepare(case, seed):
    gen = _generator(seed)
    dt = _DTYPES[case["dtype"]]
    s = {"case": case}
    if own:
        import paper_2511_16786_amd as fc
        s["fc"] = fc
    if case["kind"] == "rotary":
        B, T, d = case["batch"], case["tokens"], case["head_dim"]
        s["Q"] = torch.randn((B, T, case["q_heads"], d), generator=gen, device="cuda").to(dt)
        s["K"] = torch.randn((B, T, case["kv_heads"], d), generator=gen, device="cuda").to(dt)
        # a prompt's tokens follow each other from a place of the sequence's own
        first = torch.randint(0, max(1, case["far"] - T), (case["streams"], B, 1), generator=gen, device="cuda")
        s["positions"] = (first + torch.arange(T, device="cuda") // (1 + torch.arange(case["streams"], device="cuda"))[:, None, None]).to(torch.int32)
        f, magnitude = _frequencies(case)
        s["magnitude"] = magnitude
        s["frequencies"] = torch.tensor(f, dtype=torch.float64, device="cuda")
        s["stream"] = torch.repeat_interleave(torch.arange(case["streams"], device="cuda"), torch.tensor(_sections(case), device="cuda"))
        s["Q_out"], s["K_out"] = torch.empty_like(s["Q"]), torch.empty_like(s["K"])
        if own:
            s["plan"] = s["fc"].rotary_plan(case["rotary_dim"], theta=1.0e6, interleaved=case["interleaved"],
                                            scaling=case["scaling"], factor=case["factor"], original_tokens=32768,
                                            sections=_sections(case) if case["streams"] > 1 else None)
        return s
    B, L, H, N, d, ps = (case[k] for k in ("batch", "layers", "kv_heads", "tokens", "head_dim", "page"))
    rows = _rows(case, gen)
    grown = case["kind"] == "pages" and case["add"] > 0
    most = -(-(N + case.get("add", 0)) // ps)                          # pages that a unit's table has room for: any layer may keep all rows
    need = (-(-rows // ps)).repeat_interleave(H, 1).reshape(-1)        # pages of the units
    total = int(need.sum())
    spare = B * L * H * (1 + (case["add"] if grown else 0) // ps)
    free = torch.randperm(total + spare, generator=gen, device="cuda").to(torch.int32)
    at = torch.arange(most, device="cuda")
    first = torch.cumsum(need, 0) - need
    table = torch.where(at < need[:, None], free[(first[:, None] + at).clamp(max=total + spare - 1)], -1).view(B, L, H, most)
    s.update(num_pages=total + spare, free=free)
    if case["kind"] == "pages":
        s["rows"] = rows.to(torch.int32) if grown else torch.zeros((B, L), dtype=torch.int32, device="cuda")
        s["add"] = torch.full((B, L), case["add"], dtype=torch.int32, device="cuda") if grown else rows.to(torch.int32)
        s["cursor"] = torch.full((1,), total if grown else 0, dtype=torch.int64, device="cuda")
        s["table"] = table.contiguous() if grown else torch.full_like(table, -1)
        s["slots"] = torch.empty((B, L * H * case["add"] if grown else int(rows[0].sum()) * H), dtype=torch.int64, device="cuda")
        s["rows_out"], s["cursor_out"] = torch.empty_like(s["rows"]), torch.empty_like(s["cursor"])
        return s
    s["table"] = table.contiguous()
    s["pages"] = torch.zeros((total + spare, ps // 16 * 17 * d), dtype=torch.uint8, device="cuda")
    if case["kind"] == "store" and case["step"]:
        last = rows - 1                                                # the row that a step adds
        page = table.gather(3, (last // ps)[:, :, None, None].expand(B, L, H, 1))[..., 0].long()
        s["slots"] = (page * ps + (last % ps)[:, :, None]).reshape(B, L * H)
    elif case["kind"] != "attend":
        s["slots"] = _packed_slots(rows, table, ps, H)
    if case["kind"] == "store":
        R = s["slots"].shape[1]
        s["K"], s["V"] = _values((B, R, d), gen, dt), _values((B, R, d), gen, dt)
        s["K_out"], s["V_out"] = torch.empty_like(s["K"]), torch.empty_like(s["V"])
    elif case["kind"] == "gather":
        s["K"], s["V"] = _values((B, L, H, N, d), gen, dt), _values((B, L, H, N, d), gen, dt)
        # mean squared deviations: many alike, with a long tail
        s["scores"] = torch.rand((B, L, H, N), generator=gen, device="cuda").clamp(min=1e-6).log().neg().square() * 0.02
        s["rows"] = rows.to(torch.int32)
        s["offsets"] = torch.cat((torch.zeros((B, 1), dtype=torch.int64, device="cuda"), torch.cumsum(H * rows, 1)), 1)
        kept = H * int(rows[0].sum())
        s["kept"] = kept
        s["idx"] = torch.empty((B, kept), dtype=torch.int32, device="cuda")
        s["K_out"] = torch.empty((B, kept, d), dtype=dt, device="cuda")
        s["V_out"] = torch.empty_like(s["K_out"])
        if own:
            s["desc"] = s["fc"].describe(s["K"])
    else:
        n = (total + spare) * ps
        _write(s["pages"], torch.arange(n, device="cuda"), _values((n, d), gen, torch.float32), _values((n, d), gen, torch.float32))
        if case["holes"]:                                              # layers without rows, and pages that are gone
            rows = torch.where(torch.rand((B, L), generator=gen, device="cuda") < 0.15, 0, rows)
            s["table"] = torch.where(torch.rand(table.shape, generator=gen, device="cuda") < 0.1, -1, table).contiguous()
        s["rows"] = rows.to(torch.int32)
        s["Q"] = torch.randn((B, L, H * case["group"], d), generator=gen, device="cuda").to(dt)
        s["out"] = torch.empty((B, L, H * case["group"], d), dtype=torch.float32, device="cuda")
    return s


def _packed_slots(rows, table, ps, H):
    """Slots [B, sum] of all rows, in the order of layer, head and row."""
    B, L = rows.shape
    at = torch.arange(int(rows.max()), device="cuda")
    page = table.long().gather(3, (at // ps).expand(B, L, H, -1))
    every = page * ps + at % ps
    return every[(at < rows[:, :, None, None]).expand(B, L, H, -1)].view(B, -1)


# ---- plain forms ----------------------------------------------------------------------------
def _codes(x):
    """e2m1 codes [..., d] and E [..., d / 32] of fp32 values."""
    y = x.reshape(*x.shape[:-1], -1, 32)
    top = y.abs().amax(-1)
    E = (((top.view(torch.int32) + (1 << 21)) >> 23) - 2).clamp(2, 252)
    y = y * ((254 - E) << 23).view(torch.float32)[..., None]           # 2^(127 - E)
    a = y.abs()
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = code.to(torch.uint8) + 8 * torch.signbit(y).to(torch.uint8)
    return code.reshape(x.shape), E.to(torch.uint8)


def _views(pages, d):
    """Views of the tiles' K codes, V codes, K scales and V scales."""
    t = pages.view(-1, 17 * d)
    return (t[:, :8 * d].unflatten(1, (16, d // 2)), t[:, 8 * d:16 * d].unflatten(1, (4, 16, 4, d // 32)),
            t[:, 16 * d:16 * d + d // 2].unflatten(1, (d // 32, 16)), t[:, 16 * d + d // 2:].unflatten(1, (4, d // 32, 4)))


def _write(pages, slots, K, V):
    """Rows K, V [n, d] (fp32) into the slots [n]."""
    d = K.shape[-1]
    kc, vc, ks, vs = _views(pages, d)
    tile, i = slots // 16, slots % 16
    code, E = _codes(K)
    kc[tile, i] = code[:, 0::2] | (code[:, 1::2] << 4)
    ks[tile, :, i] = E
    code, E = _codes(V)
    vc[tile, i // 4, :, i % 4] = (code[:, 0::2] | (code[:, 1::2] << 4)).unflatten(1, (16, d // 32))
    vs[tile, i // 4, :, i % 4] = E


def _value(packed, E):
    """fp32 values [..., d] of code bytes [..., d / 2] and scales [..., d / 32]."""
    code = torch.stack((packed & 15, packed >> 4), -1).flatten(-2).to(torch.int32)
    low = code & 7
    size = torch.where(low < 2, 0.5 * low, (0.5 + 0.25 * (low & 1)) * (1 << (low >> 1)))
    signed = torch.where(code > 7, -size, size).unflatten(-1, (-1, 32))
    return (signed * (E.to(torch.int32) << 23).view(torch.float32)[..., None]).flatten(-2)


def _read(pages, slots, d):
    kc, vc, ks, vs = _views(pages, d)
    tile, i = slots // 16, slots % 16
    K = _value(kc[tile, i], ks[tile, :, i])
    V = _value(vc[tile, i // 4, :, i % 4].flatten(-2), vs[tile, i // 4, :, i % 4])
    return K, V


def _turn(x, cos, sin, R, interleaved):
    out = x.float()
    a, b = (out[..., 0:R:2], out[..., 1:R:2]) if interleaved else (out[..., :R // 2], out[..., R // 2:R])
    p, q = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((p, q), -1).flatten(-2) if interleaved else torch.cat((p, q), -1)
    return torch.cat((turned, out[..., R:]), -1).to(x.dtype)


def _plain_rotary(s):
    case = s["case"]
    angle = s["positions"].double()[s["stream"]].permute(1, 2, 0) * s["frequencies"]
    cos = (angle.cos() * s["magnitude"]).float()[:, :, None]
    sin = (angle.sin() * (-s["magnitude"] if case["inverse"] else s["magnitude"])).float()[:, :, None]
    return {n: _turn(s[n], cos, sin, case["rotary_dim"], case["interleaved"]) for n in ("Q", "K")}


def _plain_pages(s):
    case = s["case"]
    B, L, H, most = s["table"].shape
    ps = case["page"]
    rows, add = s["rows"].long(), s["add"].long()
    held, want = (rows + ps - 1) // ps, (rows + add + ps - 1) // ps
    fresh = (want - held)[:, :, None].expand(B, L, H).reshape(-1)
    first = (torch.cumsum(fresh, 0) - fresh).view(B, L, H, 1) + s["cursor"]
    at = torch.arange(most, device="cuda")
    new = (at >= held[:, :, None, None]) & (at < want[:, :, None, None])
    source = first + at - held[:, :, None, None]
    table = torch.where(new, s["free"][source.clamp(0, s["num_pages"] - 1)], s["table"])
    j = torch.arange(int(add.max()), device="cuda")
    row = rows[:, :, None, None] + j
    page = table.long().gather(3, (row // ps).clamp(max=most - 1).expand(B, L, H, -1))
    slots = (page * ps + row % ps)[(j < add[:, :, None, None]).expand(B, L, H, -1)].view(B, -1)
    return {"table": table, "slots": slots, "rows": (rows + add).to(torch.int32), "cursor": s["cursor"] + fresh.sum()}


def _plain_store(s):
    case = s["case"]
    d = case["head_dim"]
    _write(s["pages"], s["slots"].view(-1), s["K"].float().view(-1, d), s["V"].float().view(-1, d))
    K, V = _read(s["pages"], s["slots"], d)
    return {"K": K.to(s["K"].dtype), "V": V.to(s["K"].dtype)}


def _plain_gather(s):
    case = s["case"]
    B, L, H, N, d = s["K"].shape
    score = s["scores"]
    if case["shared"]:                             # the heads' sum, head after head
        score = (functools.reduce(torch.add, score.unbind(2)) / H)[:, :, None].expand(B, L, H, N)
    order = torch.sort(score, dim=3, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(3, order, torch.arange(N, device="cuda").expand_as(order))
    kept = (rank < s["rows"].long()[:, :, None, None]).nonzero()
    b, l, h, token = kept.unbind(1)
    _write(s["pages"], s["slots"].view(-1), s["K"][b, l, h, token].float(), s["V"][b, l, h, token].float())
    K, V = _read(s["pages"], s["slots"], d)
    return {"idx": token.to(torch.int32).view(B, -1), "K": K.to(s["K"].dtype), "V": V.to(s["K"].dtype)}


def _plain_attend(s):
    case = s["case"]
    B, L, H, most = s["table"].shape
    d, ps, G = case["head_dim"], case["page"], case["group"]
    j = torch.arange(max(1, int(s["rows"].max())), device="cuda")
    page = s["table"].long()[..., j // ps].view(B * L * H, -1)
    ok = (j < s["rows"].view(-1, 1).repeat_interleave(H, 0)) & (page >= 0) & (page < s["num_pages"])
    K, V = _read(s["pages"], torch.where(ok, page * ps + j % ps, 0), d)
    q = s["Q"].float().view(B * L * H, G, d)
    logit = (torch.matmul(q, K.transpose(1, 2).contiguous()) / math.sqrt(d)).masked_fill(~ok[:, None], -math.inf)
    top = logit.amax(2, keepdim=True)
    p = torch.exp(logit - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(2, keepdim=True)
    out = torch.matmul(p, V) / torch.where(total == 0.0, 1.0, total)
    return out.view(B, L, H * G, d)


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        return {"rotary": _plain_rotary, "pages": _plain_pages, "store": _plain_store, "gather": _plain_gather,
                "attend": _plain_attend}[kind](s)
    fc = s["fc"]
    if kind == "rotary":
        fc.rotary(s["plan"], s["positions"], s["Q"], s["K"], Q_out=s["Q_out"], K_out=s["K_out"], inverse=case["inverse"])
        return {"Q": s["Q_out"], "K": s["K_out"]}
    ps = case["page"]
    if kind == "pages":
        fc.assign_pages(s["rows"], s["add"], ps, s["table"], s["cursor"], s["free"], slots=s["slots"],
                        rows_out=s["rows_out"], cursor_out=s["cursor_out"])
        return {"table": s["table"], "slots": s["slots"], "rows": s["rows_out"], "cursor": s["cursor_out"]}
    if kind == "attend":
        return fc.mx_decode_attention(s["Q"], s["pages"], ps, case["kv_heads"], s["rows"], s["table"],
                                      1.0 / math.sqrt(case["head_dim"]), out=s["out"])
    if kind == "store":
        fc.mx_store(s["K"], s["V"], s["slots"], s["pages"], ps)
    else:
        fc.select_gather_mx(s["K"], s["V"], s["desc"], s["scores"], s["rows"], s["offsets"], s["kept"], s["idx"],
                            s["table"], ps, s["pages"], shared=case["shared"])
    fc.mx_load(s["slots"], s["pages"], ps, s["K_out"], s["V_out"])
    out = {"K": s["K_out"], "V": s["V_out"]}
    if kind == "gather":
        out["idx"] = s["idx"]
    return out


# ---- 64 bits, from the definitions ----------------------------------------------------------
def _grid(x):
    """What the 4-bit format holds for rows [..., d] of float64 values: the nearest of its values, the even code of two."""
    y = x.reshape(*x.shape[:-1], -1, 32)
    top = y.abs().amax(-1, keepdim=True)
    power = torch.frexp(top).exponent.to(torch.float64) - 1.0          # floor of the logarithm
    power = torch.where(top == 0.0, -200.0, power) - 2.0
    power = (power + (top >= 7.0 * torch.exp2(power))).clamp(-125.0, 125.0)
    unit = torch.exp2(power)
    size = (y / unit).abs()
    # halves up to 2, whole numbers up to 4, even numbers up to 6; round() takes ties to the even multiple, as the codes do
    held = torch.where(size <= 2.0, torch.round(2.0 * size) / 2.0, torch.where(size <= 4.0, torch.round(size), 2.0 * torch.round(size / 2.0)))
    return (torch.sign(y) * held.clamp(max=6.0) * unit).reshape(x.shape)


def _exact_attend(s):
    case = s["case"]
    B, L, H, most = s["table"].shape
    d, ps, G = case["head_dim"], case["page"], case["group"]
    values = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], dtype=torch.float64, device="cuda")
    tiles = s["pages"].view(-1, 17 * d)
    out = torch.zeros((B, L, H * G, d), dtype=torch.float64, device="cuda")
    for b in range(B):
        for l in range(L):
            n = int(s["rows"][b, l])
            for h in range(H):
                j = torch.arange(n, device="cuda")
                page = s["table"][b, l, h].long()[j // ps]
                fine = (page >= 0) & (page < s["num_pages"])
                slot = (page * ps + j % ps)[fine]
                if not slot.numel():
                    continue
                t, i = (slot // 16)[:, None], (slot % 16)[:, None]
                c = torch.arange(d, device="cuda")
                part = d // 16
                kb = tiles[t, i * (d // 2) + c // 2]
                vb = tiles[t, 8 * d + i // 4 * 2 * d + c // part * (d // 8) + i % 4 * (d // 32) + c % part // 2]
                ke = tiles[t, 16 * d + c // 32 * 16 + i].double() - 127.0
                ve = tiles[t, 16 * d + d // 2 + i // 4 * (d // 8) + c // 32 * 4 + i % 4].double() - 127.0
                K = values[((kb >> (c % 2 * 4)) & 15).long()] * torch.exp2(ke)
                V = values[((vb >> (c % 2 * 4)) & 15).long()] * torch.exp2(ve)
                logit = (s["Q"][b, l, h * G:(h + 1) * G].double()[:, None] * K).sum(2) / math.sqrt(d)
                p = torch.softmax(logit, 1)
                out[b, l, h * G:(h + 1) * G] = (p[:, :, None] * V).sum(1)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "pages":
        return None
    if kind == "attend":
        return _exact_attend(s)
    if kind == "rotary":
        R, out = case["rotary_dim"], {}
        angle = s["positions"].double()[s["stream"]].movedim(0, -1) * s["frequencies"]
        turn = torch.polar(torch.full_like(angle, s["magnitude"]), -angle if case["inverse"] else angle)[:, :, None]
        for n in ("Q", "K"):
            x = s[n].double()
            pairs = x[..., :R].unflatten(-1, (R // 2, 2)) if case["interleaved"] else x[..., :R].unflatten(-1, (2, R // 2)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            z = z if case["interleaved"] else z.transpose(-1, -2)
            out[n] = torch.cat((z.reshape(*x.shape[:-1], R), x[..., R:]), -1)
        return out
    if kind == "store":
        return {"K": _grid(s["K"].double()), "V": _grid(s["V"].double())}
    B, L, H, N, d = s["K"].shape
    scores = s["scores"]
    if case["shared"]:
        whole = scores[:, :, 0].clone()
        for h in range(1, H):
            whole += scores[:, :, h]
        scores = (whole / H)[:, :, None].expand(B, L, H, N)
    key = scores.contiguous().view(torch.int32).long() * (1 << 31) + (N - torch.arange(N, device="cuda"))     # (no score is negative)
    K, V = [], []
    for b in range(B):
        for l in range(L):
            keep = torch.topk(key[b, l], int(s["rows"][b, l]), dim=1).indices.sort(1).values
            for name, rows in (("K", K), ("V", V)):
                rows.append(_grid(s[name][b, l].double().gather(1, keep[:, :, None].expand(-1, -1, d))).reshape(-1, d))
    return {"K": torch.cat(K).view(B, -1, d), "V": torch.cat(V).view(B, -1, d), "idx": None}


def work(case):
    """Every input read once, every output written once; the rows of a cache in four bits take 17/16 bytes a column, K and V together."""
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "rotary":
        values = case["batch"] * case["tokens"] * (case["q_heads"] + case["kv_heads"]) * case["head_dim"]
        return {"bytes": 2 * values * e + 4 * case["streams"] * case["batch"] * case["tokens"],
                "flops": 3 * values * case["rotary_dim"] // case["head_dim"]}
    B, L, H, N, d, ps = (case[k] for k in ("batch", "layers", "kv_heads", "tokens", "head_dim", "page"))
    kept = B * H * max(L, int(case["rho"] * L * N))
    if case["kind"] == "pages":
        slots = B * L * H * case["add"] if case["add"] else kept
        return {"bytes": 12 * B * L + 8 * slots + 8 * -(-slots // ps) + 16, "flops": 0}
    if case["kind"] == "attend":
        q = B * L * H * case["group"] * d
        return {"bytes": kept * d * 17 // 16 + q * (e + 4), "flops": 4 * kept * case["group"] * d}
    rows = B * L * H if case["kind"] == "store" and case["step"] else kept
    moved = rows * (4 * d * e + 2 * (d * 17 // 16) + 8)                # in, into the cache, out of it, out
    if case["kind"] == "gather":
        moved += 4 * B * L * H * N + 4 * rows
    return {"bytes": moved, "flops": 2 * rows * d}
