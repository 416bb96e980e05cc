"""Workloads and plain forms of the 8-bit serving operators.

Four operators surround the block-wise FP8 projections of a decoder layer that is served with an 8-bit paged KV cache:

  norm     h = x + r in bf16, n = RMSNorm(h) * gain, and n in E4M3 codes with one scale per row and 128 channels (what
           pd_gemm_fp8_blockwise takes) or one per row (what pd_gemm_fp8 takes)
  append   rotary position rotation of the q and k heads of fresh projection rows; q is stored, k and v go to the pages of
           their sequences as E4M3 codes with one power-of-two scale per page and head, which grows with the page's tokens
  decode   attention of one query token per sequence over that cache
  prefill  causal attention of the fresh rows of every request over that cache (an optional cached prefix and themselves)

`run` computes them in their plain form (elementary torch operations in fp32), or, where `own` is set, by the library's
calls.  `exact` is the definition in 64 bits, written apart from the plain form.
"""
import math
import random

import torch

own = False  # True: run() makes the library's calls

E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
MIN_EXP, MAX_EXP = -117, 120  # exponents of a page scale
THETA = 1e4
EPS = 1e-6

# Head shapes and widths are those of this repository's configurations: 8B (32 / 8 heads of 128, width 4096), 70B
# (64 / 8 heads of 128, width 8192) and tiny (8 / 2 heads of 64, width 512).
SHAPES = {"8b": (32, 8, 128, 4096), "70b": (64, 8, 128, 8192), "tiny": (8, 2, 64, 512)}


def listed():
    return [
        # the norm in front of a projection of one decode step of a single user: latency alone
        {"name": "norm-1x4096", "op": "norm", "rows": 1, "d": 4096, "group": 128, "norm_out": False},
        # a decode batch of the 70B width that also keeps the bf16 norm (for an unquantised head), one scale per row
        {"name": "norm-200x8192-row", "op": "norm", "rows": 200, "d": 8192, "group": 0, "norm_out": True},
        # a prefill pass of one 4096-token prompt and a bit, 8B width
        {"name": "norm-4099x4096", "op": "norm", "rows": 4099, "d": 4096, "group": 128, "norm_out": False},
        # one user's decode step: a single token joins a half filled page
        {"name": "append-1-token", "op": "append", "shape": "8b", "page": 64, "n_req": 1, "new": 1, "new_hi": 1, "kv": 2090,
         "kv_hi": 2090, "lens": 1},
        # a decode batch at mixed lengths: every sequence at another place of its page
        {"name": "append-256-tokens", "op": "append", "shape": "8b", "page": 64, "n_req": 256, "new": 1, "new_hi": 1, "kv": 0,
         "kv_hi": 575, "lens": 2},
        # prompts and chunks that start and end inside pages
        {"name": "append-prompts", "op": "append", "shape": "8b", "page": 64, "n_req": 5, "new": 700, "new_hi": 4100, "kv": 0,
         "kv_hi": 1000, "lens": 3},
        # one long conversation: few rows, a long axis
        {"name": "decode-1x32768", "op": "decode", "shape": "8b", "page": 64, "n_req": 1, "new": 1, "new_hi": 1, "kv": 32767,
         "kv_hi": 32767, "lens": 4},
        # a small batch at mixed lengths in small pages, group of 8
        {"name": "decode-24-ragged", "op": "decode", "shape": "70b", "page": 16, "n_req": 24, "new": 1, "new_hi": 1, "kv": 100,
         "kv_hi": 4351, "lens": 5},
        # the throughput batch of the benchmark
        {"name": "decode-256x2304", "op": "decode", "shape": "8b", "page": 64, "n_req": 256, "new": 1, "new_hi": 1, "kv": 2000,
         "kv_hi": 2303, "lens": 6},
        # short chunks (a few drafted or resumed tokens per user) over cached prefixes, small heads
        {"name": "prefill-16x23-tiny", "op": "prefill", "shape": "tiny", "page": 32, "n_req": 16, "new": 1, "new_hi": 23, "kv": 0,
         "kv_hi": 1500, "lens": 7},
        # chunked prefill: 512-token chunks and a bit, long cached prefixes, group of 8
        {"name": "prefill-chunks", "op": "prefill", "shape": "70b", "page": 64, "n_req": 4, "new": 480, "new_hi": 530, "kv": 3000,
         "kv_hi": 8200, "lens": 8},
        # one whole prompt that has just been appended
        {"name": "prefill-4096", "op": "prefill", "shape": "8b", "page": 64, "n_req": 1, "new": 4096, "new_hi": 4096, "kv": 0,
         "kv_hi": 0, "lens": 9},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "append", "decode", "prefill"])
    if op == "norm":
        group = rng.choice([0, 128])
        return {"op": op, "rows": _log(rng, 1, 4099), "d": 128 * rng.randint(1, 32) if group else 16 * rng.randint(1, 256),
                "group": group, "norm_out": rng.random() < 0.5}
    shape, page = rng.choice(["8b", "70b", "tiny"]), rng.choice([16, 32, 64, 128])
    c = {"op": op, "shape": shape, "page": page, "lens": rng.randrange(1 << 30)}
    if op == "append":
        if rng.random() < 0.5:
            c |= {"n_req": _log(rng, 1, 256), "new": 1, "new_hi": 1, "kv": 0, "kv_hi": rng.randint(0, 575)}
        else:
            new = _log(rng, 1, 3000 if shape != "70b" else 1400)
            c |= {"n_req": rng.randint(1, 4), "new": max(0, new // 3), "new_hi": new, "kv": 0, "kv_hi": rng.randint(0, 1000)}
    elif op == "decode":
        kv = _log(rng, 1, 32767)
        c |= {"n_req": min(_log(rng, 1, 256), max(1, 500_000 // kv)), "new": 1, "new_hi": 1, "kv": rng.choice([0, kv // 2, kv]), "kv_hi": kv}
    else:
        new, n_req = _log(rng, 1, 1000 if shape != "70b" else 500), rng.randint(1, 4)
        c |= {"n_req": n_req, "new": rng.choice([0, new // 2, new]), "new_hi": new, "kv": 0, "kv_hi": _log(rng, 1, 5000)}
    return c


def lengths(case):
    """(tokens cached before the call, fresh tokens) of every request.  A decode query counts among the cached ones: it sits
    at position kv and attends to kv + 1 entries."""
    r = random.Random(case["lens"])
    kv = [r.randint(case["kv"], case["kv_hi"]) for _ in range(case["n_req"])]
    new = [r.randint(case["new"], case["new_hi"]) for _ in range(case["n_req"])]
    if sum(new) == 0:
        new[0] = 1
    return kv, new


def work(case):
    if case["op"] == "norm":
        n, d = case["rows"] * case["d"], case["d"]
        scales = n // 128 if case["group"] else case["rows"]
        return {"bytes": n * (2 + 2 + 2 + 1 + (2 if case["norm_out"] else 0)) + 2 * d + 4 * scales, "flops": 8 * n}
    hq, hkv, hd, _ = SHAPES[case["shape"]]
    kv, new = lengths(case)
    t, page = sum(new), case["page"]
    if case["op"] == "append":
        pages = sum((k + n - 1) // page - k // page + 1 for k, n in zip(kv, new) if n)
        rope = (max(k + n for k, n in zip(kv, new)) - min(kv)) if t > len(new) else len({k for k in kv})
        return {"bytes": t * (hq + 2 * hkv) * hd * 2 + t * hq * hd * 2 + t * 2 * hkv * hd + pages * hkv * 2 * 4 + min(rope, t) * hd * 4,
                "flops": t * (hq + hkv) * hd * 3 + t * 4 * hkv * hd}
    if case["op"] == "decode":
        keys = sum(k + 1 for k in kv)
        pages = sum(k // page + 1 for k in kv)
        return {"bytes": keys * hkv * hd * 2 + pages * (hkv * 8 + 4) + t * hq * hd * 4, "flops": 4 * keys * hq * hd}
    keys = sum(k + n for k, n in zip(kv, new) if n)
    pages = sum(-(-(k + n) // page) for k, n in zip(kv, new) if n)
    pairs = sum(k * n + n * (n + 1) // 2 for k, n in zip(kv, new))
    return {"bytes": keys * hkv * hd * 2 + pages * (hkv * 8 + 4) + t * hq * hd * 4, "flops": 4 * pairs * hq * hd}


# ------------------------------------------------------------------------------------------------------------- inputs
def _pow2_scale(amax):
    """The smallest power of two s with amax <= 448 s, exponent kept within MIN_EXP .. MAX_EXP."""
    m, e = torch.frexp(amax)
    e = torch.where(m > 0.875, e - 8, e - 9)  # 448 = 0.875 * 2^9
    e = torch.where(amax > 0, e, torch.full_like(e, MIN_EXP)).clamp(MIN_EXP, MAX_EXP)
    return torch.ldexp(torch.ones_like(amax, dtype=torch.float32), e)


def _pool(gen, n_pages, hkv, page, hd, written):
    """Codes and scales of n_pages random pages; `written`[n_pages] rows of each hold tokens, the others uninitialised
    memory, as which NaN codes stand."""
    x = torch.randn((n_pages, hkv, page, hd), generator=gen, device="cuda")
    x *= torch.exp(0.7 * torch.randn((n_pages, hkv, 1, 1), generator=gen, device="cuda"))
    keep = (torch.arange(page, device="cuda") < written[:, None])[:, None, :, None]
    s = _pow2_scale(torch.where(keep, x.abs(), torch.zeros((), device="cuda")).amax(dim=(2, 3)))
    x = torch.where(keep, x / s[:, :, None, None], torch.full((), float("nan"), device="cuda"))
    return x.to(E4M3).view(torch.uint8), s


def _rope_table(n, hd):
    """(cos, sin) of every position and pair, angles in 64 bits."""
    inv = THETA ** (-torch.arange(0, hd, 2, dtype=torch.float64, device="cuda") / hd)
    a = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * inv
    return torch.stack([torch.cos(a), torch.sin(a)], dim=-1).float().contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"] == "norm":
        rows, d = case["rows"], case["d"]
        s = {"case": case, "gain": (1 + 0.02 * torch.randn(d, generator=gen, device="cuda")).bfloat16(),
             "x": torch.randn((rows, d), generator=gen, device="cuda").bfloat16(),
             "r": (2 * torch.randn((rows, d), generator=gen, device="cuda")).bfloat16()}
        s["h"] = torch.empty_like(s["x"])
        s["n"] = torch.empty_like(s["x"]) if case["norm_out"] else None
        s["codes"] = torch.empty((rows, d), dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty((rows, d // 128) if case["group"] else (rows,), device="cuda")
        return s
    hq, hkv, hd, d = SHAPES[case["shape"]]
    page = case["page"]
    kv, new = lengths(case)
    append = case["op"] == "append"
    # tokens in the cache when the call begins, and after it
    before = kv if append else [k + n for k, n in zip(kv, new)]
    after = [k + n for k, n in zip(kv, new)]
    counts = [max(1, -(-a // page)) for a in after]
    width = max(counts) + 2
    n_pages = sum(counts) + 3  # a few pages of the pool are free
    order = random.Random(seed).sample(range(n_pages), n_pages)
    table, written, at = [], [0] * n_pages, 0
    for b, n in zip(before, counts):
        ids = order[at:at + n]
        at += n
        for i, p in enumerate(ids):
            written[p] = min(page, max(0, b - i * page))
        table.append(ids + [-1] * (width - n))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    w = i32(written)
    s = {"case": case, "page": page, "shape": (hq, hkv, hd), "table": i32(table), "kv": i32(kv), "kv_host": kv,
         "max_kv": max(after), "n_req": len(kv), "tokens": sum(new), "n_pages": n_pages}
    s["k"], s["k_scale"] = _pool(gen, n_pages, hkv, page, hd, w)
    s["v"], s["v_scale"] = _pool(gen, n_pages, hkv, page, hd, w)
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    s["cu"], s["cu_host"] = i32(cu), cu
    s["decode_rows"] = case["new_hi"] == 1 and case["new"] == 1
    if append:
        # key channels of very different size, as trained projections give them
        x = torch.randn((cu[-1], (hq + 2 * hkv), hd), generator=gen, device="cuda")
        x[:, hq:hq + hkv] *= torch.exp(0.8 * torch.randn((hkv, hd), generator=gen, device="cuda"))
        s["qkv"] = x.reshape(cu[-1], -1).bfloat16()
        s["q_out"] = torch.empty((cu[-1], hq * hd), dtype=torch.bfloat16, device="cuda")
        s["rope"] = _rope_table(max(after), hd)
    else:
        s["q"] = torch.randn((cu[-1], hq * hd), generator=gen, device="cuda").bfloat16()
        s["out"] = torch.empty_like(s["q"])
    if own:  # the shape, the cache's description and the scratch that a program makes once
        import paper_2603_04716_b200 as pd
        s["cfg"] = pd.LayerConfig(d, hq, hkv, hd, 4 * d, rope_theta=THETA, max_pos=max(after))
        s["cache"] = pd.paged_kv_cache_struct(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"], n_pages, page, len(kv), width)
        if case["op"] == "decode":
            s["ws_bytes"] = pd.pd_paged_decode_attention_workspace_bytes(s["cfg"], len(kv), s["max_kv"])
        if case["op"] == "prefill":
            s["ws_bytes"] = pd.pd_paged_prefill_attention_workspace_bytes(s["cfg"], len(kv), s["max_kv"])
        if not append:
            s["ws"] = torch.empty(max(256, s["ws_bytes"]), dtype=torch.uint8, device="cuda")
    return s


# -------------------------------------------------------------------------------------------------------- plain forms
def _norm_plain(s):
    group = s["case"]["group"]
    h = (s["x"].float() + s["r"].float()).bfloat16()
    f = h.float()
    y = f * torch.rsqrt(f.square().mean(dim=-1, keepdim=True) + EPS) * s["gain"].float()
    blocks = y.view(y.shape[0], -1, group) if group else y[:, None]
    amax = blocks.abs().amax(dim=-1)
    scales = torch.where(amax > 0, amax / E4M3_MAX, torch.ones_like(amax))
    codes = (blocks / scales[..., None]).clamp(-E4M3_MAX, E4M3_MAX).view_as(y).to(E4M3)
    return {"sum": h, "norm": y.bfloat16() if s["n"] is not None else None, "codes": codes, "scales": scales if group else scales[:, 0]}


def _append_plain(s):
    hq, hkv, hd = s["shape"]
    page, t, n_pages = s["page"], s["tokens"], s["n_pages"]
    cu = s["cu"].long()
    req = torch.searchsorted(cu[1:], torch.arange(t, device="cuda"), right=True)
    pos = s["kv"].long()[req] + torch.arange(t, device="cuda") - cu[req]
    x = s["qkv"].float().view(t, hq + 2 * hkv, hd)
    cs = s["rope"][pos]
    c, sn = cs[:, None, :, 0], cs[:, None, :, 1]
    lo, hi = x[:, :hq + hkv, :hd // 2], x[:, :hq + hkv, hd // 2:]
    rot = torch.cat([lo * c - hi * sn, hi * c + lo * sn], dim=-1)
    s["q_out"].copy_(rot[:, :hq].reshape(t, -1))
    pages, off = s["table"].long()[req, pos // page], pos % page
    first = torch.full((n_pages,), page, device="cuda").scatter_reduce(0, pages, off, "amin")
    old_rows = torch.arange(page, device="cuda") < first[:, None]
    touched = (first < page)[:, None]
    for codes, scale, vals in ((s["k"], s["k_scale"], rot[:, hq:]), (s["v"], s["v_scale"], x[:, hq + hkv:])):
        amax = torch.zeros((n_pages, hkv), device="cuda").index_reduce(0, pages, vals.abs().amax(dim=-1), "amax")
        need = _pow2_scale(amax)
        old = torch.where((first == 0)[:, None], torch.zeros_like(scale), scale)  # an empty page has no scale yet
        fresh = torch.where(touched, torch.maximum(old, need), scale)
        ratio = torch.where(touched & (old > 0), old / fresh, torch.ones_like(old))
        again = (ratio < 1)[:, :, None, None] & old_rows[:, None, :, None]
        at, head = torch.nonzero(ratio < 1, as_tuple=True)
        moved = (codes[at, head].view(E4M3).float() * ratio[at, head, None, None]).to(E4M3).view(torch.uint8)
        codes[at, head] = torch.where(again[at, head], moved, codes[at, head])
        new = (vals / fresh[pages][..., None]).to(E4M3).view(torch.uint8)
        codes[pages, :, off] = new
        scale.copy_(fresh)
    return {"q": s["q_out"], "k": s["k"].view(E4M3), "v": s["v"].view(E4M3), "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _gathered(s, codes, scale):
    """[n_req, Hkv, S, hd] fp32 of every page that the table names (unused entries repeat page 0 and are masked later)."""
    hq, hkv, hd = s["shape"]
    ids = s["table"].long()[:, :-(-s["max_kv"] // s["page"])].clamp(min=0)
    x = codes[ids].view(E4M3).float() * scale[ids][..., None, None]
    return x.permute(0, 2, 1, 3, 4).reshape(ids.shape[0], hkv, -1, hd)


def _softmax_plain(scores, seen):
    scores = torch.where(seen, scores, torch.full((), -math.inf, device="cuda"))
    p = torch.exp(scores - scores.amax(dim=-1, keepdim=True))
    return p / p.sum(dim=-1, keepdim=True)


def _decode_plain(s):
    hq, hkv, hd = s["shape"]
    k, v = _gathered(s, s["k"], s["k_scale"]), _gathered(s, s["v"], s["v_scale"])
    seen = torch.arange(k.shape[2], device="cuda") <= s["kv"][:, None]
    v = torch.where(seen[:, None, :, None], v, torch.zeros((), device="cuda"))
    q = s["q"].float().view(-1, hkv, hq // hkv, hd)
    p = _softmax_plain(q @ k.transpose(2, 3) / math.sqrt(hd), seen[:, None, None])
    s["out"].copy_((p @ v).reshape(s["n_req"], -1))
    return s["out"]


def _prefill_plain(s):
    hq, hkv, hd = s["shape"]
    t, cu = s["tokens"], s["cu"].long()
    req = torch.searchsorted(cu[1:], torch.arange(t, device="cuda"), right=True)
    row = torch.arange(t, device="cuda") - cu[req]
    most = max(b - a for a, b in zip(s["cu_host"], s["cu_host"][1:]))
    q = torch.zeros((s["n_req"], most, hq * hd), device="cuda")
    q[req, row] = s["q"].float()
    q = q.view(s["n_req"], most, hkv, hq // hkv, hd).permute(0, 2, 3, 1, 4).reshape(s["n_req"], hkv, -1, hd)
    k, v = _gathered(s, s["k"], s["k_scale"]), _gathered(s, s["v"], s["v_scale"])
    keys = torch.arange(k.shape[2], device="cuda")
    end = s["kv"].long() + (cu[1:] - cu[:-1])
    held = keys < end[:, None]
    k = torch.where(held[:, None, :, None], k, torch.zeros((), device="cuda"))
    v = torch.where(held[:, None, :, None], v, torch.zeros((), device="cuda"))
    seen = keys <= (s["kv"].long()[:, None] + torch.arange(most, device="cuda"))[..., None]
    scores = (q @ k.transpose(2, 3) / math.sqrt(hd)).view(s["n_req"], hkv, hq // hkv, most, -1)
    p = _softmax_plain(scores, seen[:, None, None])
    o = (p.view(s["n_req"], hkv, -1, p.shape[-1]) @ v).view(s["n_req"], hkv, hq // hkv, most, hd).permute(0, 3, 1, 2, 4)
    s["out"].copy_(o.reshape(s["n_req"], most, -1)[req, row])
    return s["out"]


# ----------------------------------------------------------------------------------------------------- the library's calls
def _own(s):
    import paper_2603_04716_b200 as pd
    op, case = s["case"]["op"], s["case"]
    if op == "norm":
        pd.pd_add_rmsnorm_fp8(s["x"], case["rows"], case["d"], s["gain"], s["codes"], s["scales"], residual=s["r"], sum_out=s["h"],
                              norm_out=s["n"], eps=EPS, group=case["group"])
        return {"sum": s["h"], "norm": s["n"], "codes": s["codes"].view(E4M3), "scales": s["scales"]}
    hq, hkv, hd = s["shape"]
    if op == "append":
        if s["decode_rows"]:
            pd.pd_paged_kv_append(s["cfg"], s["qkv"], (hq + 2 * hkv) * hd, s["q_out"], s["rope"], s["cache"], s["kv"], s["n_req"])
        else:
            pd.pd_paged_kv_append(s["cfg"], s["qkv"], (hq + 2 * hkv) * hd, s["q_out"], s["rope"], s["cache"], s["kv"], s["n_req"],
                                  cu_seqlens_dev=s["cu"], cu_seqlens_host=s["cu_host"])
        return {"q": s["q_out"], "k": s["k"].view(E4M3), "v": s["v"].view(E4M3), "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if op == "decode":
        pd.pd_paged_decode_attention(s["cfg"], s["q"], hq * hd, s["out"], s["kv"], s["n_req"], s["max_kv"], s["cache"], s["ws"], s["ws_bytes"])
    else:
        pd.pd_paged_prefill_attention(s["cfg"], s["q"], hq * hd, s["out"], s["cu"], s["cu_host"], s["kv"], s["kv_host"], s["cache"],
                                      s["ws"], s["ws_bytes"])
    return s["out"]


def run(state):
    if own:
        return _own(state)
    return {"norm": _norm_plain, "append": _append_plain, "decode": _decode_plain, "prefill": _prefill_plain}[state["case"]["op"]](state)


# --------------------------------------------------------------------------------------------------------------- exact
def _e4m3_values():
    """The 256 values of the format: sign, four exponent bits with bias 7, three mantissa bits, S.1111.111 is NaN."""
    out = []
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out.append(math.nan if e == 15 and m == 7 else -v if c & 128 else v)
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def _e4m3_round(x):
    """float64 -> nearest value of the format, ties to the even step."""
    a = x.abs().clamp(max=E4M3_MAX)
    e = torch.floor(torch.log2(a.clamp(min=2.0 ** -30))).clamp(-6, 8)
    step = torch.exp2(e - 3)
    return torch.copysign(torch.round(a / step) * step, x)


def _exact_attention(q, k, v, first):
    """Rows q[n, Hq, hd] at positions first, first + 1, ... over k, v [S, Hkv, hd]."""
    n, hq, hd = q.shape
    g = hq // k.shape[1]
    out = torch.empty_like(q)
    seen = torch.arange(k.shape[0], device="cuda") <= (first + torch.arange(n, device="cuda"))[:, None]
    for h in range(hq):
        sc = (q[:, h] @ k[:, h // g].T) * hd ** -0.5
        sc = sc.masked_fill(~seen, -math.inf)
        out[:, h] = torch.softmax(sc, dim=-1) @ v[:, h // g]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        h = (s["x"].double() + s["r"].double()).bfloat16().double()
        y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + EPS) * s["gain"].double()
        g = case["group"] or case["d"]
        b = y.reshape(case["rows"], case["d"] // g, g)
        sc = b.abs().amax(-1) / E4M3_MAX
        sc = sc.masked_fill(sc == 0, 1.0)
        codes = _e4m3_round(b / sc[..., None]).reshape(case["rows"], case["d"])
        return {"sum": h, "norm": y if case["norm_out"] else None, "codes": codes, "scales": sc.reshape(s["scales"].shape)}
    hq, hkv, hd = s["shape"]
    page, table, cu = s["page"], s["table"].tolist(), s["cu_host"]
    vals = _e4m3_values()
    if case["op"] != "append":
        out = torch.empty((cu[-1], hq * hd), dtype=torch.float64, device="cuda")
        for r in range(s["n_req"]):
            a, b, first = cu[r], cu[r + 1], s["kv_host"][r]
            if a == b:
                continue
            total = first + b - a
            ids = torch.tensor(table[r][:-(-total // page)], device="cuda")
            k, v = ((vals[s[c][ids].long()] * s[c + "_scale"][ids].double()[..., None, None]).transpose(1, 2).reshape(-1, hkv, hd)[:total]
                    for c in ("k", "v"))
            out[a:b] = _exact_attention(s["q"][a:b].double().view(-1, hq, hd), k, v, first).reshape(b - a, -1)
        return out
    held = {c: vals[s[c].long()] for c in ("k", "v")}
    scale = {c: s[c + "_scale"].double() for c in ("k", "v")}
    x = s["qkv"].double().view(-1, hq + 2 * hkv, hd)
    q_out = torch.empty((cu[-1], hq, hd), dtype=torch.float64, device="cuda")
    freq = torch.tensor([THETA ** (-2.0 * i / hd) for i in range(hd // 2)], dtype=torch.float64, device="cuda")
    for r in range(s["n_req"]):
        a, b, first = cu[r], cu[r + 1], s["kv_host"][r]
        ang = torch.arange(first, first + b - a, dtype=torch.float64, device="cuda")[:, None] * freq
        z = torch.complex(x[a:b, :hq + hkv, :hd // 2], x[a:b, :hq + hkv, hd // 2:]) * torch.polar(torch.ones_like(ang), ang)[:, None]
        z = torch.cat([z.real, z.imag], -1)
        q_out[a:b] = z[:, :hq]
        new = {"k": z[:, hq:], "v": x[a:b, hq + hkv:]}
        for i in range(first // page, (first + b - a - 1) // page + 1 if b > a else 0):
            lo, hi, p = max(first, i * page), min(first + b - a, (i + 1) * page), table[r][i]
            for c in ("k", "v"):
                rows = new[c][lo - first:hi - first].transpose(0, 1)  # [Hkv, tokens, hd]
                am = rows.abs().amax(dim=(1, 2))
                need = torch.exp2(torch.ceil(torch.log2(am.clamp(min=1e-300) / E4M3_MAX)).clamp(MIN_EXP, MAX_EXP))
                had = scale[c][p] if lo > i * page else torch.zeros_like(need)
                sc = torch.maximum(had, need)
                if lo > i * page:
                    old = held[c][p, :, :lo - i * page]
                    held[c][p, :, :lo - i * page] = _e4m3_round(old * (had / sc)[:, None, None])
                held[c][p, :, lo - i * page:hi - i * page] = _e4m3_round(rows / sc[:, None, None])
                scale[c][p] = sc
    return {"q": q_out.reshape(cu[-1], -1), "k": held["k"], "v": held["v"], "k_scale": scale["k"], "v_scale": scale["v"]}
