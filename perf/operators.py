"""Measured cases of the operators that decode over a paged cache, and their plain forms.

Three operators, in the order in which a decoding layer runs them:
  append   qcf_page_append: new keys and values into their pages, rotated on the way, queries rotated beside them
  attn     qcf_page_attn: attention of the newest tokens over every page of their request
  sparse   qcf_page_select, then qcf_page_attn over the pages that it keeps

With `own` false the calls are elementary torch operations in float32 (page scores and angles in float64), with `own` true
the library's.  A request's tokens are scattered over a pool of pages that is a quarter larger than they need, as it is after
some requests came and went.  Keys carry a slowly changing topic along a direction that queries share, so that attention
is spread unevenly over the pages, as it is over retrieved text.
"""
from __future__ import annotations

import math
import random
from typing import Dict, List, Optional

import torch

own = False

DEVICE = "cuda:0"
# query heads, KV heads, head dim, rotary base, dtype
SHAPES = {
    "tiny": (4, 2, 64, 10000.0, "f32"),
    "8b": (32, 8, 128, 500000.0, "bf16"),
    "70b": (64, 8, 128, 500000.0, "bf16"),
    "head64": (32, 8, 64, 500000.0, "bf16"),
}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def _case(name, kind, shape, requests, tokens, page, **kw) -> dict:
    """tokens: least and largest number of tokens of a request (append: of the rows that it gets; held_lo, held_hi: what it has)."""
    c = {"name": name, "kind": kind, "shape": shape, "requests": requests, "lo": tokens[0], "hi": tokens[1], "page": page,
         "style": 0, "order": "token", "new": 1, "layout": 0}
    c.update(kw)
    return c


def listed() -> List[dict]:
    return [
        # one decoding step of a small batch: a row for each request, nothing but latency
        _case("append_step_8", "append", "8b", 8, (1, 1), 16, held_lo=300, held_hi=4000),
        # drafts of the validation model: a few rows each, interleaved pairs, pages that begin and end inside
        _case("append_f32_drafts", "append", "tiny", 13, (1, 9), 32, held_lo=0, held_hi=900, style=1),
        # a short prompt with narrow heads behind what the request holds already
        _case("append_head64_731", "append", "head64", 1, (731, 731), 64, held_lo=45, held_hi=45),
        # the fused contexts of a batch go into pages: the largest append
        _case("append_batch_32k", "append", "8b", 16, (1000, 3000), 16, held_lo=0, held_hi=0),
        # the first token after a short question over three passages
        _case("attn_1x731", "attn", "8b", 1, (731, 731), 16),
        # a validation run in float32
        _case("attn_f32_5x600", "attn", "tiny", 5, (17, 600), 32, style=1),
        # a ragged batch of retrieval prompts, the middle of the range
        _case("attn_16x4k", "attn", "8b", 16, (1000, 8192), 16),
        # four drafted tokens for each of a few requests on the wide layer, some of them padding
        _case("attn_drafts_8x6001", "attn", "70b", 8, (2000, 6001), 64, new=4, padded=0.2),
        # a single very long context: the whole card works on one token
        _case("attn_1x128k", "attn", "8b", 1, (131071, 131071), 64, order="head"),
        # a full serving batch: the largest pass over the cache
        _case("attn_64x8k", "attn", "8b", 64, (4096, 12288), 16),
        # a very long context of which each head keeps a fraction of the pages
        _case("sparse_1x128k", "sparse", "8b", 1, (131071, 131071), 16, keep=256, first=1, last=2),
        # a serving batch of long contexts, narrow selection
        _case("sparse_32x16k", "sparse", "8b", 32, (8192, 24576), 16, keep=96, first=1, last=2),
    ]


def _log_int(rng: random.Random, lo: int, hi: int) -> int:
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _drawn(rng: random.Random) -> dict:
    kind = rng.choices(["append", "attn", "sparse"], [3, 5, 3])[0]
    shape = rng.choices(["8b", "70b", "head64", "tiny"], [4, 2, 2, 1])[0]
    most = 8 if shape == "tiny" else 64
    requests = _log_int(rng, 1, most)
    c = _case("", kind, shape, requests, (1, 1), rng.choice([16, 16, 32, 64, 128]),
              style=int(rng.random() < 0.25), order=rng.choice(["token", "token", "head"]), layout=rng.randrange(1 << 20))
    if kind == "append":
        rows = 1 if rng.random() < 0.4 else _log_int(rng, 1, 2048)
        c["lo"], c["hi"] = max(1, rows // 3), rows
        held = 0 if rng.random() < 0.3 else _log_int(rng, 1, 4096)
        c["held_lo"], c["held_hi"] = held // 2, held
        return c
    tokens = _log_int(rng, 1, 2048 if shape == "tiny" else 131072)
    c["hi"] = tokens
    c["lo"] = max(1, int(tokens * rng.uniform(0.1, 1.0)))
    if kind == "attn":
        c["new"] = rng.choice([1, 1, 1, 2, 3, 5, 8])
        c["padded"] = rng.choice([0.0, 0.25])
    else:
        pages = (tokens + c["page"] - 1) // c["page"]
        c["keep"] = _log_int(rng, 4, max(4, min(512, pages // 2 + 1)))
        c["first"], c["last"] = rng.randint(0, 1), rng.randint(1, 3)
    return c


def draw(rng: random.Random) -> dict:
    """One more case of the same ranges, no larger than the full serving batch."""
    limit = next(work(c)["bytes"] for c in listed() if c["name"] == "attn_64x8k")
    while True:
        c = _drawn(rng)
        c.pop("name")
        # (the plain form pads a batch to its longest request)
        if work(c)["bytes"] <= 0.9 * limit and c["requests"] * c["hi"] <= 64 * 12288:
            return c


# ------------------------------------------------------------------ layouts (of the case alone)

def _lengths(case: dict) -> List[int]:
    rng = random.Random(case["layout"])
    return [rng.randint(case["lo"], case["hi"]) for _ in range(case["requests"])]


def _held(case: dict) -> List[int]:
    rng = random.Random(case["layout"] + 1)
    return [rng.randint(case["held_lo"], case["held_hi"]) for _ in range(case["requests"])]


def _seen(case: dict, lens: List[int]) -> List[List[int]]:
    """Tokens that each new row sees; 0 for a row that only fills up the batch."""
    rng = random.Random(case["layout"] + 2)
    n = case["new"]
    return [[0 if i > 0 and rng.random() < case.get("padded", 0.0) else max(0, t - n + 1 + i) for i in range(n)] for t in lens]


def _pages(tokens: int, page: int) -> int:
    return (tokens + page - 1) // page


# ------------------------------------------------------------------ inputs

class _Draws:
    def __init__(self, case: dict, seed: int):
        self.g = torch.Generator(device=DEVICE).manual_seed(seed)
        self.H, self.Hkv, self.D, self.base, dt = SHAPES[case["shape"]]
        self.G = self.H // self.Hkv
        self.dt = DTYPES[dt]
        self.u = torch.sign(self.normal(self.Hkv, self.D, dtype=torch.float32))      # shared by keys and queries of a group

    def normal(self, *size, dtype=None) -> torch.Tensor:
        return torch.randn(*size, generator=self.g, device=DEVICE, dtype=dtype or self.dt)

    def keys(self, n: int, run: int = 48) -> torch.Tensor:
        k = self.normal(n, self.Hkv, self.D)
        topic = self.normal(n // run + 1, dtype=torch.float32).repeat_interleave(run)[:n]
        return k.add_((0.25 * topic[:, None, None] * self.u).to(self.dt))

    def queries(self, *lead: int) -> torch.Tensor:
        q = self.normal(*lead, self.H, self.D)
        return q.add_((0.5 * self.u.repeat_interleave(self.G, dim=0)).to(self.dt))


def _pool(case: dict, r: _Draws, n_pages: int) -> torch.Tensor:
    """[n_pages, page, H_kv, d], the heads of a token or the tokens of a head next to each other."""
    if case["order"] == "head":
        return torch.empty(n_pages, r.Hkv, case["page"], r.D, dtype=r.dt, device=DEVICE).transpose(1, 2)
    return torch.empty(n_pages, case["page"], r.Hkv, r.D, dtype=r.dt, device=DEVICE)


def _cache(case: dict, r: _Draws, capacity: List[int], filled: List[int]) -> dict:
    """Pools with `filled` tokens of each request, a table with pages for `capacity`, and the bounds of what is filled."""
    page, B = case["page"], len(capacity)
    counts = [_pages(c, page) for c in capacity]
    width = max(counts)
    n_pages = max(1, sum(counts) + sum(counts) // 4)
    order = torch.randperm(n_pages, generator=r.g, device=DEVICE)
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEVICE)
    fill = torch.zeros(n_pages, dtype=torch.int64, device=DEVICE)
    at = 0
    slot0 = torch.arange(width, device=DEVICE) * page
    for b, n in enumerate(counts):
        mine = order[at:at + n]
        at += n
        table[b, :n] = mine.int()
        fill[mine] = (filled[b] - slot0[:n]).clamp(0, page)
    k, v = _pool(case, r, n_pages), _pool(case, r, n_pages)
    # (in parts of 64 MB or so, so that drawing does not need the pool in float32 as well)
    step = max(1, (1 << 24) // (page * r.Hkv * r.D))
    lo = torch.empty(n_pages, r.Hkv, 2, r.D, dtype=r.dt, device=DEVICE)
    for p in range(0, n_pages, step):
        n = min(step, n_pages - p)
        part = r.keys(n * page).view(n, page, r.Hkv, r.D)
        k[p:p + n] = part
        v[p:p + n] = r.normal(n, page, r.Hkv, r.D)
        held = (torch.arange(page, device=DEVICE) < fill[p:p + n, None])[:, :, None, None]
        lo[p:p + n, :, 0] = part.masked_fill(~held, math.inf).amin(1)
        lo[p:p + n, :, 1] = part.masked_fill(~held, -math.inf).amax(1)
    lo.masked_fill_((fill == 0)[:, None, None, None], 0.0)
    return {"k": k, "v": v, "bounds": lo, "table": table, "page": page, "width": width}


def _library(case: dict, s: dict) -> None:
    """The descriptors and workspaces that a program keeps."""
    from paper_2604_08585_amd import binding as qb
    from paper_2604_08585_amd import inputs
    H, Hkv, D, base, dt = SHAPES[case["shape"]]
    s["desc"] = qb.make_desc(inputs.LayerShape(H * D, H, Hkv, D, base, dt, case["style"]))
    c = s["cache"]
    s["pages"] = qb.page_cache(c["k"], c["v"], c["bounds"], c["table"])
    ws = lambda n: torch.empty(n, dtype=torch.uint8, device=DEVICE) if n else None
    if case["kind"] == "sparse":
        s["ws_select"] = ws(qb.qcf_page_select_workspace_bytes(s["desc"], s["pages"], s["B"], s["new"], s["keep"]))
    if case["kind"] != "append":
        s["ws_attn"] = ws(qb.qcf_page_attn_workspace_bytes(s["desc"], s["pages"], s["B"], s["new"], s.get("keep", 0)))


def prepare(case: dict, seed: int) -> dict:
    r = _Draws(case, seed)
    B, lens = case["requests"], _lengths(case)
    s: Dict = {"kind": case["kind"], "B": B, "H": r.H, "Hkv": r.Hkv, "D": r.D, "base": r.base, "style": case["style"],
               "new": case["new"]}
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEVICE)
    if case["kind"] == "append":
        held = _held(case)
        s["cache"] = _cache(case, r, [h + n for h, n in zip(held, lens)], held)
        off = [0]
        for n in lens:
            off.append(off[-1] + n)
        s["rows"] = off[-1]
        s["row_off"] = torch.tensor(off, dtype=torch.int64, device=DEVICE)
        s["lens"] = i32(held)
        s["pos"] = i32([h + i for h, n in zip(held, lens) for i in range(n)])
        # the rows of one product: queries, keys and values side by side
        qkv = r.normal(s["rows"], (r.H + 2 * r.Hkv) * r.D)
        cut = [r.H * r.D, r.Hkv * r.D, r.Hkv * r.D]
        s["q"], s["k"], s["v"] = (t.unflatten(1, (-1, r.D)) for t in qkv.split(cut, 1))
        s["q_out"] = torch.zeros(s["rows"], r.H, r.D, dtype=r.dt, device=DEVICE)
    else:
        s["cache"] = _cache(case, r, lens, lens)
        s["seen"] = i32(_seen(case, lens))
        s["q"] = r.queries(B, case["new"])
        s["o"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(B, case["new"], r.H, dtype=torch.float32, device=DEVICE)
        if case["kind"] == "sparse":
            s["keep"], s["first"], s["last"] = case["keep"], case["first"], case["last"]
            s["list"] = torch.zeros(B, case["new"], r.Hkv, case["keep"], dtype=torch.int32, device=DEVICE)
    if own:
        _library(case, s)
    return s


# ------------------------------------------------------------------ the library's calls

def _run_own(s: dict):
    from paper_2604_08585_amd import binding as qb
    c = s["cache"]
    if s["kind"] == "append":
        qb.qcf_page_append(s["desc"], s["pages"], s["B"], s["q"], s["k"], s["v"], s["row_off"], s["rows"], s["lens"], s["pos"],
                           s["q_out"])
        return {"k": c["k"], "v": c["v"], "bounds": c["bounds"], "q": s["q_out"]}
    if s["kind"] == "attn":
        qb.qcf_page_attn(s["desc"], s["pages"], s["B"], s["new"], s["q"], s["seen"], None, 0, s["o"], s["lse"], s["ws_attn"])
        return {"o": s["o"], "lse": s["lse"]}
    qb.qcf_page_select(s["desc"], s["pages"], s["B"], s["new"], s["q"], s["seen"], s["keep"], s["first"], s["last"], s["list"],
                       s["ws_select"])
    qb.qcf_page_attn(s["desc"], s["pages"], s["B"], s["new"], s["q"], s["seen"], s["list"], s["keep"], s["o"], s["lse"],
                     s["ws_attn"])
    return {"pages": s["list"], "o": s["o"], "lse": s["lse"]}


# ------------------------------------------------------------------ the plain forms

def _rotated(x: torch.Tensor, pos: torch.Tensor, base: float, style: int) -> torch.Tensor:
    """Rows [M, heads, d] turned by their positions; the angles in float64, the products in float32."""
    d = x.shape[-1]
    theta = base ** (torch.arange(d // 2, device=x.device, dtype=torch.float64) * (-2.0 / d))
    phi = pos.double()[:, None] * theta
    cos, sin = phi.cos().float()[:, None], phi.sin().float()[:, None]
    x = x.float()
    a, b = (x[..., :d // 2], x[..., d // 2:]) if style == 0 else (x[..., 0::2], x[..., 1::2])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    return torch.cat([ra, rb], -1) if style == 0 else torch.stack([ra, rb], -1).flatten(-2)


def _run_append(s: dict):
    c, page = s["cache"], s["cache"]["page"]
    rows = torch.arange(s["rows"], device=DEVICE)
    req = torch.searchsorted(s["row_off"], rows, right=True) - 1
    token = s["lens"][req].long() + rows - s["row_off"][req]
    at, slot = c["table"][req, token // page].long(), token % page
    k = _rotated(s["k"], s["pos"], s["base"], s["style"]).to(c["k"].dtype)
    c["k"][at, slot] = k
    c["v"][at, slot] = s["v"]
    s["q_out"].copy_(_rotated(s["q"], s["pos"], s["base"], s["style"]))
    # a page that gets its first slot here starts anew
    bounds = c["bounds"]
    fresh = at[slot == 0]
    bounds[fresh, :, 0] = math.inf
    bounds[fresh, :, 1] = -math.inf
    where = at[:, None, None].expand_as(k)
    bounds[:, :, 0] = bounds[:, :, 0].float().scatter_reduce(0, where, k.float(), "amin").to(k.dtype)
    bounds[:, :, 1] = bounds[:, :, 1].float().scatter_reduce(0, where, k.float(), "amax").to(k.dtype)
    return {"k": c["k"], "v": c["v"], "bounds": bounds, "q": s["q_out"]}


def _keep(s: dict) -> torch.Tensor:
    """The pages that are kept, ascending, -1 behind the last: [B, new, H_kv, keep]."""
    c, page, G = s["cache"], s["cache"]["page"], s["H"] // s["Hkv"]
    count = (s["seen"].long() + page - 1) // page                                      # [B, new]
    p = torch.arange(c["width"], device=DEVICE)
    q = s["q"].double().unflatten(2, (s["Hkv"], G)).transpose(1, 2)                    # [B, H_kv, new, G, d]
    scores = []
    for b in range(s["B"]):
        lo, hi = c["bounds"][c["table"][b].clamp(min=0).long()].double().permute(1, 2, 3, 0).unbind(1)   # [H_kv, d, pages]
        x = q[b].flatten(1, 2)
        dots = x.clamp(max=0.0) @ lo.contiguous() + x.clamp(min=0.0) @ hi.contiguous()
        scores.append(dots.unflatten(1, (s["new"], G)).amax(2).transpose(0, 1))        # [new, H_kv, pages]
    score = torch.stack(scores).float()
    n = count[:, :, None, None]
    forced = (p < s["first"]) | (p >= n - s["last"])
    score = score.masked_fill(forced, math.inf).masked_fill(p >= n, -math.inf)
    best = score.sort(dim=-1, descending=True, stable=True).indices[..., :s["keep"]]
    best = torch.where(best < n, best, c["width"]).sort(-1).values
    out = torch.full_like(s["list"], -1)
    out[..., :best.shape[-1]] = torch.where(best < c["width"], best, -1).int()
    return out


def _attend(s: dict, tokens: torch.Tensor, visible: torch.Tensor):
    """tokens [B, H_kv, L]: rows of the pools; visible [B, H_kv, new, L]."""
    c, G, B, n = s["cache"], s["H"] // s["Hkv"], s["B"], s["new"]
    page = c["page"]
    heads = torch.arange(s["Hkv"], device=DEVICE)[:, None]
    q = s["q"].float().unflatten(2, (s["Hkv"], G)).permute(0, 2, 1, 3, 4).flatten(2, 3)       # [B, H_kv, new * G, d]
    o = torch.empty_like(s["o"])
    lse = torch.empty_like(s["lse"])
    for b in range(B):
        k = c["k"][tokens[b] // page, tokens[b] % page, heads].float()                 # [H_kv, L, d]
        logits = (q[b] @ k.transpose(1, 2)) * s["D"] ** -0.5
        logits = logits.masked_fill(~visible[b].repeat_interleave(G, 1), -math.inf)
        top = logits.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
        e = (logits - top).exp()
        total = e.sum(-1, keepdim=True)
        v = c["v"][tokens[b] // page, tokens[b] % page, heads].float()
        out = (e @ v) / total.clamp(min=1e-30)
        o[b] = out.unflatten(1, (n, G)).permute(1, 0, 2, 3).flatten(1, 2).to(o.dtype)
        lse[b] = (top + total.log()).squeeze(-1).unflatten(1, (n, G)).permute(1, 0, 2).flatten(1)
    return o, lse


def run(s: dict):
    if own:
        return _run_own(s)
    if s["kind"] == "append":
        return _run_append(s)
    c, page = s["cache"], s["cache"]["page"]
    slots = torch.arange(page, device=DEVICE)
    if s["kind"] == "attn":
        t = torch.arange(c["width"] * page, device=DEVICE)
        rows = (c["table"].clamp(min=0).long()[:, :, None] * page + slots).flatten(1)                # [B, L]
        o, lse = _attend(s, rows[:, None].expand(-1, s["Hkv"], -1), (t < s["seen"][:, :, None])[:, None].expand(-1, s["Hkv"], -1, -1))
        return {"o": o, "lse": lse}
    kept = _keep(s)
    lists = kept[:, 0].clamp(min=0).long()                                                           # (one new row to a request)
    phys = c["table"].long()[torch.arange(s["B"], device=DEVICE)[:, None, None], lists].clamp(min=0)
    rows = (phys[..., None] * page + slots).flatten(2)
    t = (lists[..., None] * page + slots).flatten(2)
    shown = (t < s["seen"][:, :, None]) & (kept[:, 0] >= 0).repeat_interleave(page, -1)
    o, lse = _attend(s, rows, shown[:, :, None])
    return {"pages": kept, "o": o, "lse": lse}


# ------------------------------------------------------------------ definitions in 64 bits

def _exact_append(s: dict):
    c, page, D = s["cache"], s["cache"]["page"], s["D"]
    k, v, bounds = c["k"].double(), c["v"].double(), c["bounds"].double()
    pair = torch.arange(D // 2, device=DEVICE, dtype=torch.float64)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE),
                       s["pos"].double()[:, None, None] * torch.exp(-2.0 * pair / D * math.log(s["base"])))
    i = torch.arange(D // 2, device=DEVICE)
    first, second = (i, i + D // 2) if s["style"] == 0 else (2 * i, 2 * i + 1)

    def turned(x):
        z = torch.complex(x[..., first].double(), x[..., second].double()) * turn
        y = torch.empty(x.shape, dtype=torch.float64, device=DEVICE)
        y[..., first], y[..., second] = z.real, z.imag
        return y

    kr = turned(s["k"])
    off, held = s["row_off"].tolist(), s["lens"].tolist()
    for b in range(s["B"]):
        t, end = held[b], held[b] + off[b + 1] - off[b]
        while t < end:
            p, n = int(c["table"][b, t // page]), min(end, (t // page + 1) * page) - t
            m = off[b] + t - held[b]
            k[p, t % page:t % page + n] = kr[m:m + n]
            v[p, t % page:t % page + n] = s["v"][m:m + n].double()
            lo, hi = kr[m:m + n].amin(0), kr[m:m + n].amax(0)
            if t % page:
                lo, hi = torch.minimum(lo, bounds[p, :, 0]), torch.maximum(hi, bounds[p, :, 1])
            bounds[p, :, 0], bounds[p, :, 1] = lo, hi
            t += n
    return {"k": k, "v": v, "bounds": bounds, "q": turned(s["q"])}


def exact(case: dict, seed: int) -> Optional[dict]:
    s = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(s)
    c, page, G, D = s["cache"], s["cache"]["page"], s["H"] // s["Hkv"], s["D"]
    o, lse = torch.zeros(s["o"].shape, dtype=torch.float64, device=DEVICE), torch.full(s["lse"].shape, -math.inf, dtype=torch.float64,
                                                                                       device=DEVICE)
    pages = torch.full_like(s["list"], -1) if case["kind"] == "sparse" else None
    seen = s["seen"].tolist()
    for b in range(s["B"]):
        most = max(seen[b])
        mine = c["table"][b, :_pages(most, page)].long()
        for g in range(s["Hkv"]):
            kb = vb = None
            if pages is None:
                kb, vb = c["k"][mine, :, g].double().flatten(0, 1), c["v"][mine, :, g].double().flatten(0, 1)
            for i in range(s["new"]):
                n = seen[b][i]
                if n == 0:
                    continue
                q = s["q"][b, i, g * G:(g + 1) * G].double()
                if pages is None:
                    kk, vv = kb[:n], vb[:n]
                else:
                    count = _pages(n, page)
                    edge = c["bounds"][mine[:count], g].double()
                    # (page by page and element by element the larger of both products, in parts)
                    top = torch.cat([(q[:, None, None] * e).amax(2).sum(-1).amax(0) for e in edge.split(256)]).float()
                    top[:s["first"]] = math.inf
                    top[max(0, count - s["last"]):] = math.inf
                    chosen = torch.argsort(-top, stable=True)[:s["keep"]].sort().values
                    pages[b, i, g, :chosen.numel()] = chosen.int()
                    shown = (chosen[:, None] * page + torch.arange(page, device=DEVICE)).flatten() < n
                    kk = c["k"][mine[chosen], :, g].double().flatten(0, 1)[shown]
                    vv = c["v"][mine[chosen], :, g].double().flatten(0, 1)[shown]
                logits = (kk @ q.t()) / math.sqrt(D)                                   # [tokens, G]
                z = torch.logsumexp(logits, 0)
                lse[b, i, g * G:(g + 1) * G] = z
                o[b, i, g * G:(g + 1) * G] = torch.exp(logits - z).t() @ vv
    out = {"o": o, "lse": lse}
    return {"pages": pages, **out} if pages is not None else out


def work(case: dict) -> dict:
    H, Hkv, D, _, dt = SHAPES[case["shape"]]
    size, page, lens = SIZE[dt], case["page"], _lengths(case)
    B, n = case["requests"], case["new"]
    if case["kind"] == "append":
        rows, bounds = sum(lens), 0
        for h, m in zip(_held(case), lens):
            touched = (h + m - 1) // page - h // page + 1
            bounds += (touched + (1 if h % page else 0)) * 2 * Hkv * D * size
        return {"bytes": rows * ((2 * H + 4 * Hkv) * D * size + 4) + bounds + 12 * B, "flops": 3 * rows * (H + Hkv) * D}
    seen = _seen(case, lens)
    rows = B * n * H
    nbytes = rows * (2 * D * size + 4)
    flops = 0
    for req in seen:
        if case["kind"] == "attn":
            nbytes += max(req) * 2 * Hkv * D * size + 4 * _pages(max(req), page)
            flops += sum(4 * H * D * t for t in req)
            continue
        for t in req:
            count = _pages(t, page)
            kept = min(count, case["keep"])
            tokens = max(0, kept * page - (count * page - t))
            nbytes += count * (2 * Hkv * D * size + 4) + tokens * 2 * Hkv * D * size + 8 * Hkv * case["keep"]
            flops += 4 * H * D * (count + tokens)
    return {"bytes": nbytes, "flops": flops}
