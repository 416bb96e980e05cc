"""Workloads and plain forms of the operators around the 4-bit paged KV cache.

Five operators serve the attention half of a decoder layer whose q and k heads are normalised, rotated by scaled positions, and
cached in 4 bits:

  table   (cos, sin) of rotary angles for a range of positions, frequencies scaled for contexts longer than the trained one
  norm    RMSNorm of every q and k head and the rotation of its first features, halves or neighbours paired
  append  the same for fresh projection rows; q is stored, k and v go to the pages of their sequences in 4 bits: E2M1 codes,
          one E4M3 scale per 16 features, one power of two per head.  The fresh rows are read back from their pages, as the
          attention of the same rows takes them
  read    cached positions of sequences read back as bf16
  decode  attention of one or several query tokens per sequence over that cache

`run` computes them in their plain form (elementary torch operations), or, where `own` is set, by the library's calls.  `exact`
is the definition in 64 bits, written apart from the plain form.  Keys are normalised, rotated and quantised in 64 bits in the
plain form, too: a code is a decision, and one next to a border has to fall on the same side everywhere.
"""
import math
import random

import torch

own = False  # True: run() makes the library's calls

EPS = 1e-6
THETA = 1e4
STEPS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # magnitudes of E2M1 codes 0 .. 7
GROUP = 16  # features that share a scale

# Head shapes are those of this repository's configurations: 8B (32 / 8 heads of 128), 70B (64 / 8 heads of 128) and tiny (8 / 2
# heads of 64).
SHAPES = {"8b": (32, 8, 128), "70b": (64, 8, 128), "tiny": (8, 2, 64)}
SCALINGS = ("none", "linear", "base", "turns", "index")


def listed():
    return [
        # the table of a short-context replica at start-up
        {"name": "table-1000", "op": "table", "first": 0, "n": 1000, "rot": 64, "scaling": "none", "factor": 1.0, "trained": 4096},
        # the same for a context 32 times the trained one
        {"name": "table-131072-scaled", "op": "table", "first": 0, "n": 131072, "rot": 128, "scaling": "turns", "factor": 32.0,
         "trained": 4096},
        # a decode batch of the 70B heads, half of each head rotated, neighbours paired
        {"name": "norm-200-pairs", "op": "norm", "shape": "70b", "rows": 200, "rot": 64, "pairs": True, "gains": True, "far": 40000},
        # a prefill pass of one 4096-token prompt and a bit
        {"name": "norm-4099", "op": "norm", "shape": "8b", "rows": 4099, "rot": 128, "pairs": False, "gains": True, "far": 4099},
        # one user's decode step
        {"name": "append-1-token", "op": "append", "shape": "8b", "page": 64, "rot": 128, "pairs": False, "gains": True, "n_req": 1,
         "new": 1, "new_hi": 1, "kv": 2090, "kv_hi": 2090, "lens": 1},
        # a decode batch at mixed lengths
        {"name": "append-256-tokens", "op": "append", "shape": "8b", "page": 64, "rot": 128, "pairs": False, "gains": True,
         "n_req": 256, "new": 1, "new_hi": 1, "kv": 0, "kv_hi": 575, "lens": 2},
        # prompts and chunks that start and end inside pages
        {"name": "append-prompts", "op": "append", "shape": "8b", "page": 64, "rot": 128, "pairs": False, "gains": True, "n_req": 5,
         "new": 700, "new_hi": 4100, "kv": 0, "kv_hi": 1000, "lens": 3},
        # the prefix of one resumed conversation
        {"name": "read-1x1500", "op": "read", "shape": "tiny", "page": 32, "n_req": 1, "kv": 1500, "kv_hi": 1500, "lens": 4},
        # prefixes of a chunked prefill batch, ragged
        {"name": "read-24-ragged", "op": "read", "shape": "8b", "page": 16, "n_req": 24, "kv": 900, "kv_hi": 8200, "lens": 5},
        # one long conversation: few rows, a long axis
        {"name": "decode-1x32768", "op": "decode", "shape": "8b", "page": 64, "n_req": 1, "new": 1, "kv": 32767, "kv_hi": 32767,
         "lens": 6},
        # a small batch at mixed lengths in small pages, group of 8, one drafted token beside the newest
        {"name": "decode-24-ragged-x2", "op": "decode", "shape": "70b", "page": 16, "n_req": 24, "new": 2, "kv": 100, "kv_hi": 4351,
         "lens": 7},
        # the throughput batch of the benchmark
        {"name": "decode-256x2304", "op": "decode", "shape": "8b", "page": 64, "n_req": 256, "new": 1, "kv": 2000, "kv_hi": 2303,
         "lens": 8},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["table", "norm", "append", "read", "decode"])
    if op == "table":
        return {"op": op, "first": rng.choice([0, rng.randint(1, 1 << 20)]), "n": _log(rng, 1, 131072), "rot": 16 * rng.randint(1, 8),
                "scaling": rng.choice(SCALINGS), "factor": rng.uniform(1, 40), "trained": rng.choice([2048, 4096, 8192])}
    shape, page = rng.choice(list(SHAPES)), rng.choice([16, 32, 64, 128])
    hd = SHAPES[shape][2]
    turn = {"rot": 16 * rng.randint(1, hd // 16), "pairs": rng.random() < 0.5, "gains": rng.random() < 0.7}
    if op == "norm":
        return {"op": op, "shape": shape, "rows": _log(rng, 1, 4099 if shape != "70b" else 2000), "far": _log(rng, 8, 100_000), **turn}
    c = {"op": op, "shape": shape, "page": page, "lens": rng.randrange(1 << 30)}
    if op == "append":
        if rng.random() < 0.5:
            return {**c, **turn, "n_req": _log(rng, 1, 256), "new": 1, "new_hi": 1, "kv": 0, "kv_hi": rng.randint(0, 575)}
        new = _log(rng, 1, 3000 if shape != "70b" else 1400)
        return {**c, **turn, "n_req": rng.randint(1, 4), "new": max(0, new // 3), "new_hi": new, "kv": 0, "kv_hi": rng.randint(0, 1000)}
    if op == "read":
        kv = _log(rng, 1, 20000)
        return {**c, "n_req": min(_log(rng, 1, 100), max(1, 100_000 // kv)), "kv": rng.choice([0, kv // 2, kv]), "kv_hi": kv}
    kv = _log(rng, 1, 32760)
    return {**c, "n_req": min(_log(rng, 1, 256), max(1, 500_000 // kv)), "new": rng.choice([1, 1, 2, 3, 5]), "kv": rng.choice([0, kv // 2, kv]),
            "kv_hi": kv}


def lengths(case):
    """(tokens cached before the call, fresh tokens) of every request.  The first of a sequence's decode queries counts among
    the cached tokens: query j sits at position kv + j and attends to kv + j + 1 entries."""
    r = random.Random(case["lens"])
    kv = [r.randint(case["kv"], case["kv_hi"]) for _ in range(case["n_req"])]
    new = [r.randint(case.get("new", 0), case.get("new_hi", case.get("new", 0))) for _ in range(case["n_req"])]
    if case["op"] == "append" and sum(new) == 0:
        new[0] = 1
    if case["op"] == "read" and sum(kv) == 0:
        kv[0] = 1
    return kv, new


def work(case):
    if case["op"] == "table":
        return {"bytes": case["n"] * case["rot"] * 4, "flops": 8 * case["n"] * case["rot"]}
    hq, hkv, hd = SHAPES[case["shape"]]
    if case["op"] == "norm":
        n = case["rows"] * (hq + hkv) * hd
        return {"bytes": 4 * n + min(case["rows"], case["far"]) * case["rot"] * 4, "flops": 8 * n}
    kv, new = lengths(case)
    if case["op"] == "append":
        t = sum(new)
        fresh = t * 2 * hkv * hd
        turn = len({k + i for k, n in zip(kv, new) for i in range(n)}) * case["rot"] * 4
        # rows in, q and codes out, and the fresh values back in bf16
        return {"bytes": t * (hq + 2 * hkv) * hd * 2 + t * hq * hd * 2 + fresh * 9 // 16 + turn + fresh * 2, "flops": 8 * t * (hq + 2 * hkv) * hd}
    if case["op"] == "read":
        n = sum(kv) * 2 * hkv * hd
        return {"bytes": n * 9 // 16 + 2 * n, "flops": 2 * n}
    keys = sum(k + n for k, n in zip(kv, new))
    seen = sum(k + 1 + j for k, n in zip(kv, new) for j in range(n))
    return {"bytes": keys * hkv * hd * 2 * 9 // 16 + sum(new) * hq * hd * 4, "flops": 4 * seen * hq * hd}


# ------------------------------------------------------------------------------------------------------------- inputs
def _quantise(x):
    """Codes (0 .. 15) and scales, as values, of x [..., 16 g] in its own precision."""
    b = x.view(*x.shape[:-1], -1, GROUP)
    t = (b.abs().amax(dim=-1) / 6).clamp(max=448.0)
    # E4M3: three bits behind the leading one, steps of 2^-9 below 2^-6, ties to even
    e = (torch.frexp(t)[1] - 1).clamp(min=-6)
    step = torch.ldexp(torch.ones_like(t), e - 3)
    s = torch.round(t / step) * step
    a = torch.where(s[..., None] > 0, b.abs() / s[..., None], torch.zeros((), dtype=x.dtype, device=x.device))
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() + (a >= 3.5).byte() + (a > 5).byte())
    code = code + 8 * ((b < 0) & (code > 0)).byte()
    return code.reshape(x.shape), s


def _pack(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _e4m3_bytes(s):
    return s.float().to(torch.float8_e4m3fn).view(torch.uint8)


def _pool(gen, n_pages, hkv, page, hd, written, channels):
    """Packed codes and scales of n_pages random pages; `written`[n_pages] rows of each hold tokens, the others uninitialised
    memory, as which NaN scales stand."""
    codes = torch.randint(0, 256, (n_pages, hkv, page, hd // 2), generator=gen, device="cuda", dtype=torch.uint8)
    scales = torch.full((n_pages, hkv, page, hd // GROUP), 0x7F, device="cuda", dtype=torch.uint8)
    each = max(1, (1 << 26) // (hkv * page * hd))
    for i in range(0, n_pages, each):
        n = min(each, n_pages - i)
        x = torch.randn((n, hkv, page, hd), generator=gen, device="cuda") * channels
        x *= torch.exp(0.5 * torch.randn((n, hkv, page, 1), generator=gen, device="cuda"))
        keep = (torch.arange(page, device="cuda") < written[i:i + n, None])[:, None, :, None]
        c, s = _quantise(x)
        codes[i:i + n] = torch.where(keep, _pack(c), codes[i:i + n])
        scales[i:i + n] = torch.where(keep, _e4m3_bytes(s), scales[i:i + n])
    return codes, scales


def _scaled(case, pos):
    """Table rows of positions `pos`, in 64 bits, by the definition; for the inputs of the other operators."""
    return _rotary(pos, case["rot"], "none", 1.0, 4096)


def _rotary(pos, rot, scaling, factor, trained):
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    theta, m = THETA, 1.0
    if scaling == "base":
        theta = theta * factor ** (rot / max(rot - 2, 1))
    f = torch.exp(i * (-2.0 * math.log(theta) / rot))
    if scaling == "linear":
        f = f / factor
    if scaling in ("turns", "index"):
        low, high = LIMITS
        if scaling == "turns":
            keep = ((f * (trained / (2 * math.pi)) - low) / (high - low)).clamp(0, 1)
        else:
            a, b = _index_bounds(rot, trained)
            keep = 1 - ((i - a) / max(b - a, 1e-3)).clamp(0, 1)
            m = MAGNITUDE
        f = f * keep + f / factor * (1 - keep)
    a = pos.double()[:, None] * f
    return (torch.stack([torch.cos(a), torch.sin(a)], dim=-1) * m).float()


LIMITS = (1.0, 4.0)  # turns within the trained length: below the first a frequency is divided, above the second it is kept
MAGNITUDE = 1.15     # of the table where frequencies are blended by pair index


def _index_bounds(rot, trained):
    at = [rot * math.log(trained / (2 * math.pi * n)) / (2 * math.log(THETA)) for n in LIMITS]
    return max(math.floor(at[1]), 0), min(math.ceil(at[0]), rot // 2 - 1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"] == "table":
        # a replica with other positions from seed to seed
        first = case["first"] + seed % 997
        s = {"case": case, "first": first, "table": torch.empty((case["n"], case["rot"] // 2, 2), device="cuda")}
        if own:
            import paper_2603_04716_b200 as pd
            kind = {"none": pd.ROPE_SCALE_NONE, "linear": pd.ROPE_SCALE_LINEAR, "base": pd.ROPE_SCALE_BASE, "turns": pd.ROPE_SCALE_TURNS,
                    "index": pd.ROPE_SCALE_INDEX}[case["scaling"]]
            s["rope"] = pd.RopeConfig(case["rot"], THETA, kind, case["factor"], case["trained"], *LIMITS,
                                      MAGNITUDE if case["scaling"] == "index" else 1.0)
        return s
    hq, hkv, hd = SHAPES[case["shape"]]
    s = {"case": case, "shape": (hq, hkv, hd)}
    if case["op"] in ("norm", "append"):
        gain = lambda: (1 + 0.2 * torch.randn(hd, generator=gen, device="cuda")).bfloat16()  # noqa: E731
        s["q_gain"], s["k_gain"] = (gain(), gain()) if case["gains"] else (None, None)
        channels = torch.exp(0.8 * torch.randn((hkv, hd), generator=gen, device="cuda"))  # key channels of very different size
        rows = case["rows"] if case["op"] == "norm" else sum(lengths(case)[1])
        x = torch.randn((rows, hq + 2 * hkv, hd), generator=gen, device="cuda")
        x[:, hq:hq + hkv] *= channels
        s["qkv"] = x.reshape(rows, -1).bfloat16()
        s["q_out"] = torch.empty((rows, hq * hd), dtype=torch.bfloat16, device="cuda")
    if case["op"] == "norm":
        s["pos"] = torch.randint(0, case["far"], (case["rows"],), generator=gen, device="cuda", dtype=torch.int32)
        s["rope"] = _scaled(case, torch.arange(case["far"], device="cuda"))
        s["k_out"] = torch.empty((case["rows"], hkv * hd), dtype=torch.bfloat16, device="cuda")
        if own:
            import paper_2603_04716_b200 as pd
            s["cfg"] = pd.LayerConfig(hq * hd, hq, hkv, hd, hq * hd)
            s["turn"] = _transform(pd, s)
        return s
    page = case["page"]
    kv, new = lengths(case)
    append = case["op"] == "append"
    held = kv if append or case["op"] == "read" else [k + n for k, n in zip(kv, new)]  # when the call begins
    after = [k + n for k, n in zip(kv, new)]
    counts = [max(1, -(-a // page)) for a in after]
    width = max(counts) + 2
    n_pages = sum(counts) + 3  # a few pages of the pool are free
    order = random.Random(seed).sample(range(n_pages), n_pages)
    table, written, at = [], [0] * n_pages, 0
    for b, n in zip(held, counts):
        ids = order[at:at + n]
        at += n
        for i, p in enumerate(ids):
            written[p] = min(page, max(0, b - i * page))
        table.append(ids + [-1] * (width - n))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    w = i32(written)
    s |= {"page": page, "table": i32(table), "kv": i32(kv), "kv_host": kv, "new_host": new, "max_kv": max(after), "n_req": len(kv)}
    channels = torch.exp(0.6 * torch.randn((hkv, 1, hd), generator=gen, device="cuda"))
    s["k"], s["k_scale"] = _pool(gen, n_pages, hkv, page, hd, w, channels)
    s["v"], s["v_scale"] = _pool(gen, n_pages, hkv, page, hd, w, torch.ones_like(channels))
    # powers of two per head, as a calibration gives them
    s["k_exp"] = torch.randint(-2, 3, (hkv,), generator=gen, device="cuda", dtype=torch.int32)
    s["v_exp"] = torch.randint(-3, 1, (hkv,), generator=gen, device="cuda", dtype=torch.int32)
    if append:
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        s["cu"], s["cu_host"], s["end"] = i32(cu), cu, i32(after)
        s["most"] = max(new)
        s["rope"] = _scaled(case, torch.arange(max(after), device="cuda"))
        s["decode_rows"] = case["new"] == 1 and case["new_hi"] == 1
        for c in ("k", "v"):
            s[c + "_back"] = torch.zeros((len(kv), hkv, s["most"], hd), dtype=torch.bfloat16, device="cuda")
    elif case["op"] == "read":
        s["zero"] = torch.zeros_like(s["kv"])
        s["most"] = max(kv)
        for c in ("k", "v"):
            s[c + "_back"] = torch.zeros((len(kv), hkv, s["most"], hd), dtype=torch.bfloat16, device="cuda")
    else:
        s["q"] = torch.randn((len(kv) * case["new"], hq * hd), generator=gen, device="cuda").bfloat16()
        s["out"] = torch.empty_like(s["q"])
    if own:  # the descriptions and the scratch that a program makes once
        import paper_2603_04716_b200 as pd
        s["cfg"] = pd.LayerConfig(hq * hd, hq, hkv, hd, hq * hd)
        s["cache"] = pd.paged_kv4_cache_struct(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"], n_pages, page, len(kv), width,
                                               k_exp=s["k_exp"], v_exp=s["v_exp"])
        if append:
            s["turn"] = _transform(pd, s)
        if case["op"] == "decode":
            s["ws_bytes"] = pd.pd_paged_kv4_decode_attention_workspace_bytes(s["cfg"], len(kv), case["new"], s["max_kv"])
            s["ws"] = torch.empty(max(256, s["ws_bytes"]), dtype=torch.uint8, device="cuda")
        else:
            s["back"] = pd.kv_cache_struct(s["k_back"], s["v_back"], len(kv), s["most"])
    return s


def _transform(pd, s):
    return pd.qk_transform_struct(s["rope"], s["rope"].shape[0], s["case"]["rot"], pd.ROPE_PAIRS if s["case"]["pairs"] else pd.ROPE_HALVES,
                                  q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS)


# -------------------------------------------------------------------------------------------------------- plain forms
def _table_plain(s):
    c = s["case"]
    s["table"].copy_(_rotary(torch.arange(s["first"], s["first"] + c["n"], device="cuda"), c["rot"], c["scaling"], c["factor"], c["trained"]))
    return s["table"]


def _turned(x, gain, cs, pairs):
    """Heads x [T, H, hd] normalised (where there is a gain) and rotated by the rows cs [T, rot / 2, 2], in the precision of x."""
    if gain is not None:
        x = x / torch.sqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * gain.to(x.dtype)
    c, sn = cs[:, None, :, 0].to(x.dtype), cs[:, None, :, 1].to(x.dtype)
    rot = 2 * cs.shape[1]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, w = a * c - b * sn, b * c + a * sn
    y = torch.stack([u, w], dim=-1).flatten(-2) if pairs else torch.cat([u, w], dim=-1)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _norm_plain(s):
    hq, hkv, hd = s["shape"]
    x = s["qkv"].float().view(-1, hq + 2 * hkv, hd)
    cs, pairs = s["rope"][s["pos"].long()], s["case"]["pairs"]
    s["q_out"].copy_(_turned(x[:, :hq], s["q_gain"], cs, pairs).flatten(1))
    s["k_out"].copy_(_turned(x[:, hq:hq + hkv], s["k_gain"], cs, pairs).flatten(1))
    return {"q": s["q_out"], "k": s["k_out"]}


def _values(codes, scales, exp):
    """fp32 values of packed codes [n, Hkv, ..., hd / 2] with their scale bytes and head exponents [Hkv] along the second axis."""
    steps = torch.tensor(STEPS + tuple(-v for v in STEPS), device="cuda")
    x = torch.stack([steps[(codes & 15).int()], steps[(codes >> 4).int()]], dim=-1).flatten(-2)
    sc = scales.view(torch.float8_e4m3fn).float()
    x = (x.view(*sc.shape, GROUP) * sc[..., None]).flatten(-2)
    return torch.ldexp(x, exp.view(1, -1, *([1] * (x.dim() - 2))))


def _rows(s, codes, scales, exp, req, pos):
    """fp32 values [n, Hkv, hd] of (request, position) pairs."""
    page = s["table"].long()[req, pos // s["page"]]
    return _values(codes[page, :, pos % s["page"]], scales[page, :, pos % s["page"]], exp)


def _append_plain(s):
    hq, hkv, hd = s["shape"]
    cu = s["cu"].long()
    at = torch.arange(s["qkv"].shape[0], device="cuda")
    req = torch.searchsorted(cu[1:], at, right=True)
    row = at - cu[req]
    pos = s["kv"].long()[req] + row
    x = s["qkv"].view(-1, hq + 2 * hkv, hd)
    cs, pairs = s["rope"][pos], s["case"]["pairs"]
    s["q_out"].copy_(_turned(x[:, :hq].float(), s["q_gain"], cs, pairs).flatten(1))
    k = _turned(x[:, hq:hq + hkv].double(), s["k_gain"], cs, pairs)
    page, off = s["table"].long()[req, pos // s["page"]], pos % s["page"]
    for c, vals in (("k", k), ("v", x[:, hq + hkv:].double())):
        code, scale = _quantise(torch.ldexp(vals, -s[c + "_exp"][:, None]))
        s[c][page, :, off] = _pack(code)
        s[c + "_scale"][page, :, off] = _e4m3_bytes(scale)
        s[c + "_back"][req, :, row] = _rows(s, s[c], s[c + "_scale"], s[c + "_exp"], req, pos).bfloat16()
    return {"q": s["q_out"], "k": s["k_back"], "v": s["v_back"]}


def _gathered(s, c):
    """[n_req, Hkv, S, hd] fp32 of every page that the table names (unused entries repeat page 0 and are masked later)."""
    hkv, hd = s["shape"][1:]
    ids = s["table"].long()[:, :-(-s["max_kv"] // s["page"])].clamp(min=0)
    x = _values(s[c][ids].flatten(0, 1), s[c + "_scale"][ids].flatten(0, 1), s[c + "_exp"])
    return x.view(*ids.shape, hkv, s["page"], hd).permute(0, 2, 1, 3, 4).reshape(ids.shape[0], hkv, -1, hd)


def _read_plain(s):
    seen = (torch.arange(s["most"], device="cuda") < s["kv"][:, None])[:, None, :, None]
    for c in ("k", "v"):
        back = s[c + "_back"]
        back.copy_(torch.where(seen, _gathered(s, c)[:, :, :s["most"]].bfloat16(), back))
    return {"k": s["k_back"], "v": s["v_back"]}


def _decode_plain(s):
    hq, hkv, hd = s["shape"]
    n, new = s["n_req"], s["case"]["new"]
    k, v = _gathered(s, "k"), _gathered(s, "v")
    keys = torch.arange(k.shape[2], device="cuda")
    held = (keys < s["kv"][:, None] + new)[:, None, :, None]
    zero = torch.zeros((), device="cuda")
    k, v = torch.where(held, k, zero), torch.where(held, v, zero)
    seen = keys <= (s["kv"][:, None] + torch.arange(new, device="cuda"))[..., None]  # [n, new, S]
    q = s["q"].float().view(n, new, hkv, hq // hkv, hd).permute(0, 2, 3, 1, 4).reshape(n, hkv, -1, hd)
    x = (q @ k.transpose(2, 3) / math.sqrt(hd)).view(n, hkv, -1, new, k.shape[2])
    x = torch.where(seen[:, None, None], x, torch.full((), -math.inf, device="cuda"))
    p = torch.exp(x - x.amax(dim=-1, keepdim=True))
    p = (p / p.sum(dim=-1, keepdim=True)).flatten(2, 3)
    s["out"].copy_((p @ v).view(n, hkv, -1, new, hd).permute(0, 3, 1, 2, 4).reshape(n * new, -1))
    return s["out"]


# ----------------------------------------------------------------------------------------------------- the library's calls
def _own(s):
    import paper_2603_04716_b200 as pd
    op = s["case"]["op"]
    if op == "table":
        pd.pd_rope_table_scaled(s["rope"], s["first"], s["case"]["n"], s["table"])
        return s["table"]
    hq, hkv, hd = s["shape"]
    n_qkv = (hq + 2 * hkv) * hd
    if op == "norm":
        pd.pd_qk_norm_rope(s["cfg"], s["turn"], s["qkv"], n_qkv, s["q_out"], hq * hd, s["k_out"], hkv * hd, s["pos"], s["case"]["rows"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "append":
        if s["decode_rows"]:
            pd.pd_paged_kv4_append(s["cfg"], s["turn"], s["qkv"], n_qkv, s["q_out"], s["cache"], s["kv"], s["n_req"])
        else:
            pd.pd_paged_kv4_append(s["cfg"], s["turn"], s["qkv"], n_qkv, s["q_out"], s["cache"], s["kv"], s["n_req"],
                                   cu_seqlens_dev=s["cu"], cu_seqlens_host=s["cu_host"])
        pd.pd_paged_kv4_read(s["cfg"], s["cache"], s["kv"], s["end"], s["n_req"], s["most"], s["back"], origin_dev=s["kv"])
        return {"q": s["q_out"], "k": s["k_back"], "v": s["v_back"]}
    if op == "read":
        pd.pd_paged_kv4_read(s["cfg"], s["cache"], s["zero"], s["kv"], s["n_req"], s["most"], s["back"])
        return {"k": s["k_back"], "v": s["v_back"]}
    pd.pd_paged_kv4_decode_attention(s["cfg"], s["q"], hq * hd, s["out"], s["kv"], s["n_req"], s["case"]["new"], s["max_kv"], s["cache"],
                                     s["ws"], s["ws_bytes"])
    return s["out"]


def run(state):
    if own:
        return _own(state)
    return {"table": _table_plain, "norm": _norm_plain, "append": _append_plain, "read": _read_plain,
            "decode": _decode_plain}[state["case"]["op"]](state)


# --------------------------------------------------------------------------------------------------------------- exact
def _code_values():
    """The 16 values of the 4-bit format: sign, two exponent bits with bias 1, one mantissa bit."""
    out = []
    for c in range(16):
        e, m = (c >> 1) & 3, c & 1
        v = m / 2 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1)
        out.append(-v if c & 8 else v)
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def _scale_values():
    """The 256 values of E4M3: sign, four exponent bits with bias 7, three mantissa bits, S.1111.111 is NaN."""
    out = []
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out.append(math.nan if e == 15 and m == 7 else -v if c & 128 else v)
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def _nearest(x, grid):
    """Non-negative x rounded to the increasing values `grid`, whose even places are the even codes; ties to those."""
    hi = torch.searchsorted(grid, x).clamp(max=len(grid) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - x, x - grid[lo]
    return torch.where((up < down) | ((up == down) & (hi % 2 == 0)), grid[hi], grid[lo])


def _exact_cached(x, exp):
    """What the cache holds of x [n, Hkv, hd], in 64 bits."""
    unit = torch.exp2(exp.double())[:, None, None]
    b = (x.reshape(*x.shape[:2], -1, GROUP)) / unit
    sc = _nearest((b.abs().amax(-1) / 6).clamp(max=448.0), _scale_values()[:127])[..., None]
    mag = torch.where(sc > 0, _nearest((b.abs() / sc.clamp(min=2.0 ** -20)).clamp(max=6.0), _code_values()[:8]), 0.0)
    return (torch.copysign(mag, b) * sc * unit).reshape(x.shape)


def _exact_turned(x, gain, ang, pairs, magnitude=1.0):
    """x [T, H, hd], angles [T, rot / 2]."""
    if gain is not None:
        x = x * (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).rsqrt() * gain.double()
    rot = 2 * ang.shape[1]
    y = x.clone()
    first = slice(0, rot, 2) if pairs else slice(0, rot // 2)
    second = slice(1, rot, 2) if pairs else slice(rot // 2, rot)
    z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.full_like(ang, magnitude), ang)[:, None]
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_angles(pos, rot, scaling="none", factor=1.0, trained=4096):
    theta = THETA * factor ** (rot / (rot - 2)) if scaling == "base" else THETA
    freq = []
    for i in range(rot // 2):
        f = theta ** (-2.0 * i / rot)
        if scaling == "linear":
            f /= factor
        if scaling in ("turns", "index"):
            low, high = LIMITS
            if scaling == "turns":
                w = (trained * f / (2 * math.pi) - low) / (high - low)
            else:
                place = lambda turns: rot / 2 * math.log(trained / (turns * 2 * math.pi), THETA)  # noqa: E731
                a, b = max(0, math.floor(place(high))), min(rot // 2 - 1, math.ceil(place(low)))
                w = 1 - (i - a) / max(b - a, 1e-3)
            w = min(1.0, max(0.0, w))
            f = w * f + (1 - w) * f / factor
        freq.append(f)
    return pos.double()[:, None] * torch.tensor(freq, dtype=torch.float64, device="cuda")


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "table":
        a = _exact_angles(torch.arange(case["n"], device="cuda") + s["first"], case["rot"], case["scaling"], case["factor"], case["trained"])
        return torch.view_as_real(torch.polar(torch.full_like(a, MAGNITUDE if case["scaling"] == "index" else 1.0), a))
    hq, hkv, hd = s["shape"]
    if case["op"] in ("norm", "append"):
        x = s["qkv"].double().view(-1, hq + 2 * hkv, hd)
    if case["op"] == "norm":
        ang = _exact_angles(s["pos"], case["rot"])
        return {"q": _exact_turned(x[:, :hq], s["q_gain"], ang, case["pairs"]).flatten(1),
                "k": _exact_turned(x[:, hq:hq + hkv], s["k_gain"], ang, case["pairs"]).flatten(1)}
    kv, new = s["kv_host"], s["new_host"]
    if case["op"] == "append":
        q = torch.empty((x.shape[0], hq, hd), dtype=torch.float64, device="cuda")
        back = {c: torch.zeros(s[c + "_back"].shape, dtype=torch.float64, device="cuda") for c in ("k", "v")}
        for r in range(s["n_req"]):
            a, b = s["cu_host"][r], s["cu_host"][r + 1]
            if a == b:
                continue
            # the table's entries are fp32 numbers, given to the call
            cs = s["rope"][kv[r]:kv[r] + b - a].double()
            mag, ang = torch.hypot(cs[..., 0], cs[..., 1]), torch.atan2(cs[..., 1], cs[..., 0])
            y = _exact_turned(x[a:b, :hq + hkv], None if s["k_gain"] is None else torch.ones(hd, device="cuda"), torch.zeros_like(ang), case["pairs"])
            gains = torch.cat([torch.ones((n, hd), device="cuda") if g is None else g.expand(n, hd) for g, n in ((s["q_gain"], hq), (s["k_gain"], hkv))])
            y = y * gains.double()
            rot = case["rot"]
            first, second = (slice(0, rot, 2), slice(1, rot, 2)) if case["pairs"] else (slice(0, rot // 2), slice(rot // 2, rot))
            z = torch.complex(y[..., first], y[..., second]) * torch.polar(mag, ang)[:, None]
            y[..., first], y[..., second] = z.real, z.imag
            q[a:b] = y[:, :hq]
            for c, rows in (("k", y[:, hq:]), ("v", x[a:b, hq + hkv:])):
                back[c][r, :, :b - a] = _exact_cached(rows, s[c + "_exp"]).transpose(0, 1)
        return {"q": q.flatten(1), **back}
    codes, scales = _code_values(), _scale_values()

    def cached(c, r, total):
        ids = s["table"][r, :-(-total // s["page"])].long()
        w = s[c][ids].long()
        v = torch.stack([codes[w % 16], codes[w // 16]], dim=-1).reshape(*w.shape[:-1], hd)
        v = v * scales[s[c + "_scale"][ids].long()].repeat_interleave(GROUP, dim=-1)
        return (v * torch.exp2(s[c + "_exp"].double())[:, None, None]).transpose(1, 2).reshape(-1, hkv, hd)[:total]

    if case["op"] == "read":
        back = {c: torch.zeros(s[c + "_back"].shape, dtype=torch.float64, device="cuda") for c in ("k", "v")}
        for r in range(s["n_req"]):
            for c in ("k", "v"):
                if kv[r]:
                    back[c][r, :, :kv[r]] = cached(c, r, kv[r]).transpose(0, 1)
        return back
    n = case["new"]
    out = torch.empty((s["n_req"], n, hq, hd), dtype=torch.float64, device="cuda")
    q = s["q"].double().view(s["n_req"], n, hq, hd)
    for r in range(s["n_req"]):
        k, v = cached("k", r, kv[r] + n), cached("v", r, kv[r] + n)
        for j in range(n):
            z = torch.einsum("ghd,sgd->ghs", q[r, j].view(hkv, -1, hd), k[:kv[r] + 1 + j]) * hd ** -0.5
            out[r, j] = torch.einsum("ghs,sgd->ghd", torch.softmax(z, dim=-1), v[:kv[r] + 1 + j]).reshape(hq, hd)
    return out.reshape(s["n_req"] * n, -1)
