"""Workloads for measuring the operators of a decoder layer around its attention, through their public entry points.

A served model's step has, around the attention over its cache, norms with the
residual's addition (``norm``), products with 4-bit weights (``product``), the
two together with 8-bit rows between them (``norm8``), and after a step of
drafted tokens their verification (``verify``).

With ``own`` false, ``run`` computes them in their plain form with elementary
torch operations in 32 bits (cumulative sums of probabilities in 64, as an
index is decided by them); with ``own`` true it calls the framework.  ``exact``
computes the definitions in 64 bits.

Sizes are those of the serving testbed that the repository's baseline notes
quote (32 query and 8 key heads of 128; 32 and 64 requests at once) and
generic ones around them.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4, "fp8": 1, "int8": 1}
CODE_MAX = {"fp8": 448.0, "int8": 127.0}
CODE_TYPE = {"fp8": torch.float8_e4m3fn, "int8": torch.int8}
SCALE_MIN = 2.0 ** -100
EPS = 1e-6

DEFAULTS = dict(rows=1, k=4096, n=4096, dtype="bf16", residual="same", kind="", group=128, zeros=False, gated=False,
                row_group=0, batch=1, drafts=4, vocab=32_000, draft=True, near=0.5)


def _full(case: dict) -> dict:
    return {**DEFAULTS, **case}


def listed() -> list:
    return [
        # one request's next token before a layer's products: latency alone
        dict(name="norm_one", op="norm", rows=1),
        # an 8K prompt's rows
        dict(name="norm_prompt", op="norm", rows=8192, k=5120),
        # packed questions of a model with an odd width, its residual stream held in 32 bits
        dict(name="norm_ragged", op="norm", rows=777, k=2051, dtype="f16", residual="f32"),
        # 32 requests' rows to 8-bit floating point and through a projection
        dict(name="norm8_step", op="norm8", rows=32, kind="fp8"),
        # three requests' rows to int8 with a scale for each group of the weights, a narrow projection
        dict(name="norm8_groups", op="norm8", rows=3, k=5120, n=1280, dtype="f16", residual="f32", kind="int8",
             group=64, row_group=64, zeros=True),
        # one request's query, key and value projection
        dict(name="product_one", op="product", rows=1, n=6144),
        # the gated pair of a feed-forward layer for one request and its three drafted tokens
        dict(name="product_gate", op="product", rows=4, k=5120, n=25_600, group=64, zeros=True, gated=True),
        # 64 requests' int8 rows through the feed-forward layer's second product
        dict(name="product_down", op="product", rows=64, k=25_600, n=5120, kind="int8"),
        # odd sizes and small groups
        dict(name="product_ragged", op="product", rows=7, k=2059, n=1003, dtype="f16", group=32, zeros=True),
        # one request's four drafted tokens
        dict(name="verify_one", op="verify", dtype="f32"),
        # 64 requests at once, a large vocabulary
        dict(name="verify_batch", op="verify", batch=64, vocab=151_936, dtype="f32"),
        # drafts that were looked up, not drawn; probabilities in 16 bits, an odd vocabulary
        dict(name="verify_lookup", op="verify", batch=24, drafts=7, vocab=50_257, dtype="bf16", draft=False),
    ]


def _log_int(rng: random.Random, lo: int, hi: int) -> int:
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng: random.Random) -> dict:
    """A case of the same ranges; drawn again where it would cost more than the largest listed one."""
    while True:
        c = _draw(rng)
        w = work(c)
        probabilities = c["batch"] * (2 * c["drafts"] + 1) * c["vocab"] if c["op"] == "verify" else 0
        if w["flops"] <= 1.67e10 and w["bytes"] <= 3.3e8 and probabilities <= 8.76e7:
            return c


def _draw(rng: random.Random) -> dict:
    op = rng.choice(["norm", "norm8", "product", "product", "verify"])
    c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "f16"]))
    if op == "norm":
        k = _log_int(rng, 512, 8192)
        c.update(rows=_log_int(rng, 1, 8192), k=k if rng.random() < 0.3 else max(64, k // 64 * 64),
                 residual=rng.choice(["same", "same", "f32", "none"]))
        return c
    if op == "verify":
        c.update(batch=_log_int(rng, 1, 64), drafts=rng.choice([1, 2, 4, 7, 8]), vocab=_log_int(rng, 1000, 151_936),
                 draft=rng.random() < 0.75, dtype=rng.choice(["f32", "f32", "bf16", "f16"]), near=rng.choice([0.2, 0.5, 1.0]))
        return c
    k, n = _log_int(rng, 256, 25_600), _log_int(rng, 128, 25_600)
    c.update(rows=_log_int(rng, 1, 64), k=k, n=n, group=rng.choice([32, 64, 128, 128]), zeros=rng.random() < 0.4,
             gated=op == "product" and rng.random() < 0.3)
    if rng.random() < 0.7:
        c.update(k=max(256, k // 128 * 128), n=max(128, n // 32 * 32))
    if c["gated"]:
        c["n"] = max(128, n // 32 * 32)
    if op == "norm8" or rng.random() < 0.4:
        c["kind"] = rng.choice(["fp8", "int8"])
    if op == "norm8":
        c["residual"] = rng.choice(["same", "f32"])
    if c.get("kind") and rng.random() < 0.3:
        c.update(k=max(256, k // 128 * 128), row_group=c["group"])
    return c


# ------------------------------------------------------------ sizes
def work(case: dict) -> dict:
    c = _full(case)
    M, K, N, e = c["rows"], c["k"], c["n"], 2
    if c["op"] == "verify":  # the row of each sequence that its last token is drawn from, of both models
        rows = 2 if c["draft"] else 1
        e = BYTES[c["dtype"]]
        return {"bytes": c["batch"] * (rows * c["vocab"] * e + c["drafts"] * (2 * e + 20) + 16),
                "flops": c["batch"] * c["vocab"] * (rows + 1)}
    kept = 0 if c["residual"] == "none" else 4 if c["residual"] == "f32" else e
    b, f = 0, 0
    if c["op"] in ("norm", "norm8"):
        b, f = M * K * (e + 2 * kept) + K * e, 6 * M * K
    if c["op"] == "norm":
        return {"bytes": b + M * K * e, "flops": f}
    groups = -(-K // c["group"])
    row = K * BYTES[c["kind"] or c["dtype"]] + (4 * (K // c["row_group"] if c["row_group"] else 1) if c["kind"] else 0)
    b += N * -(-K // 2) + N * groups * (3 if c["zeros"] else 2) + M * row * (1 if c["op"] == "product" else 2)
    return {"bytes": b + M * (N // 2 if c["gated"] else N) * e, "flops": f + 2 * M * N * K}


# ------------------------------------------------------------ inputs
def _rows(g, n: int, k: int) -> torch.Tensor:
    """Rows of a residual stream or of a product: unit normal, a few channels many times larger, as trained models have."""
    x = torch.randn(n, k, generator=g, device=DEV)
    return x * (1 + 9 * (torch.rand(k, generator=g, device=DEV) < 0.01).float())


def _encode(y: torch.Tensor, kind: str, group: int) -> tuple:
    """Codes of rows in f32 and their scales [rows, groups], one a row or one a group of columns."""
    m, k = y.shape
    parts = y.view(m, -1, group or k)
    scale = (parts.abs().amax(-1) * (1.0 / CODE_MAX[kind])).clamp_min(SCALE_MIN)
    z = (parts * scale.reciprocal()[..., None]).clamp(-CODE_MAX[kind], CODE_MAX[kind])
    return (z if kind == "fp8" else z.round()).to(CODE_TYPE[kind]).view(m, k), scale


def _weights(g, c: dict) -> dict:
    """4-bit codes [n, k / 2], the even column in the low bits, as checkpoints hold them, with a scale (and a zero)
    for each group of a row."""
    n, k = c["n"], c["k"]
    groups = -(-k // c["group"])
    codes = (torch.randn(n, k + k % 2, generator=g, device=DEV) * 2.7 + 8).round_().clamp_(0, 15).to(torch.uint8)
    scales = (0.5 + torch.rand(n, groups, generator=g, device=DEV)) / (2.7 * math.sqrt(k))
    zeros = (torch.randn(n, groups, generator=g, device=DEV) + 8).round().clamp(0, 15).to(torch.uint8)
    return dict(codes=codes[:, ::2] | (codes[:, 1::2] << 4), scales=scales.to(TYPES[c["dtype"]]),
                zeros=zeros if c["zeros"] else None)


def prepare(case: dict, seed: int) -> dict:
    c = _full(case)
    g = torch.Generator(device=DEV).manual_seed(seed)
    s, t, M, K = dict(c=c), TYPES[c["dtype"]], c["rows"], c["k"]
    if c["op"] == "verify":
        B, S, V = c["batch"], c["drafts"], c["vocab"]
        logits = torch.randn(B, S + 1, V, generator=g, device=DEV) * 3
        s["target"] = torch.softmax(logits, -1).to(t)
        if c["draft"]:
            # a smaller model's probabilities, near the target's, and tokens drawn from them
            near = logits[:, :S] + c["near"] * torch.randn(B, S, V, generator=g, device=DEV)
            s["draft"] = torch.softmax(near, -1).to(t)
            s["tokens"] = torch.multinomial(s["draft"].float().view(-1, V), 1, generator=g).view(B, S)
        else:
            s["draft"] = None
            s["tokens"] = torch.multinomial((s["target"][:, :S].float() ** 2).reshape(-1, V), 1, generator=g).view(B, S)
        s["accept"] = torch.rand(B, S, generator=g, device=DEV)
        s["final"] = torch.rand(B, generator=g, device=DEV)
        # requests near their end have fewer drafts, the first one at least none
        s["counts"] = torch.randint(S // 2, S + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        return s
    if c["op"] in ("norm", "norm8"):
        s["x"] = _rows(g, M, K).to(t)
        if c["residual"] != "none":
            kind = t if c["residual"] == "same" else torch.float32
            s["residual"] = (4 * _rows(g, M, K)).to(kind)
            s["kept"] = torch.empty_like(s["residual"])  # the stream's other buffer
        s["weight"] = (1 + 0.3 * torch.randn(K, generator=g, device=DEV)).to(t)
    if c["op"] in ("norm8", "product"):
        s.update(_weights(g, c))
    if c["op"] == "product":
        x = _rows(g, M, K)
        if c["kind"]:
            s["codes8"], s["scale8"] = _encode(x, c["kind"], c["row_group"])
        else:
            s["x"] = x.to(t)
    return s


# ------------------------------------------------------------ the framework's calls
def _handles(s: dict) -> dict:
    """What a program keeps beside its tensors: the weights as the framework lays them out, and 8-bit rows' pairs."""
    if "handles" not in s:
        from paper_2609_40247_amd import operators as O
        h = {"O": O}
        if "codes" in s:
            h["weights"] = O.Weights4(s["codes"], s["scales"], s["zeros"], k=s["c"]["k"])
        if "codes8" in s:
            h["rows"] = O.Rows8(s["codes8"], s["scale8"])
        s["handles"] = h
    return s["handles"]


def _run_own(s: dict) -> dict:
    c, h = s["c"], _handles(s)
    O, t = h["O"], TYPES[c["dtype"]]
    if c["op"] == "verify":
        tokens, accepted = O.verify_drafts(s["target"], s["tokens"], s["accept"], s["final"], draft=s["draft"],
                                           counts=s["counts"])
        return dict(tokens=tokens, accepted=accepted)
    if c["op"] == "product":
        return dict(y=O.product4(h.get("rows", s.get("x")), h["weights"], gated=c["gated"], dtype=t))
    residual = s.get("residual")
    r = dict(residual=s["kept"]) if residual is not None else {}
    y = O.norm_rows(s["x"], s["weight"], residual, eps=EPS, residual_out=s.get("kept"),
                    kind=CODE_TYPE[c["kind"]] if c["op"] == "norm8" else None, group=c["row_group"])
    if c["op"] == "norm8":
        y = O.product4(y, h["weights"], dtype=t)
    return dict(y=y, **r)


# ------------------------------------------------------------ the plain form
def _dense(s: dict) -> torch.Tensor:
    """The weights [n, k] in 32 bits."""
    c = s["c"]
    code = torch.stack([s["codes"] & 15, s["codes"] >> 4], -1).view(c["n"], -1)[:, :c["k"]].float()
    at = torch.arange(c["k"], device=DEV) // c["group"]
    zero = s["zeros"].float()[:, at] if s["zeros"] is not None else 8.0
    return (code - zero) * s["scales"].float()[:, at]


def _values(codes: torch.Tensor, scale: torch.Tensor, group: int) -> torch.Tensor:
    m, k = codes.shape
    return (codes.float().view(m, -1, group or k) * scale[..., None]).view(m, k)


def _run_plain(s: dict) -> dict:
    c = s["c"]
    t = TYPES[c["dtype"]]
    if c["op"] == "verify":
        B, S = s["tokens"].shape
        p = s["target"].gather(2, torch.cat([s["tokens"], s["tokens"][:, :1]], 1)[..., None])[:, :S, 0].double()
        q = s["draft"].gather(2, s["tokens"][..., None])[..., 0].double() if c["draft"] else torch.ones_like(p)
        t_at = torch.arange(S + 1, device=DEV)[None]
        good = (s["accept"].double() * q < p) & (t_at[:, :S] < s["counts"][:, None])
        accepted = good.long().cumprod(1).sum(1)
        b = torch.arange(B, device=DEV)
        row, all_good = s["target"][b, accepted].double(), accepted >= s["counts"]
        at = accepted.clamp_max(S - 1)
        if c["draft"]:
            other = s["draft"][b, at].double()
        else:
            other = torch.zeros_like(row).scatter_(1, s["tokens"][b, at][:, None], 1.0)
        left = torch.where(all_good[:, None], row, (row - other).clamp_min(0.0))
        left = torch.where(left.sum(1, keepdim=True) > 0, left, row)
        total = left.cumsum(1)
        above = total > s["final"].double()[:, None] * total[:, -1:]
        last = torch.where(above, torch.arange(above.shape[1], device=DEV), above.shape[1]).amin(1)
        tokens = torch.cat([s["tokens"], s["tokens"][:, :1]], 1)
        tokens = torch.where(t_at < accepted[:, None], tokens, torch.where(t_at == accepted[:, None], last[:, None], -1))
        return dict(tokens=tokens, accepted=accepted.int())
    r = {}
    if c["op"] == "product":
        x = _values(s["codes8"], s["scale8"], c["row_group"]) if c["kind"] else s["x"].float()
    else:
        h = s["x"].float()
        if c["residual"] != "none":
            h = h + s["residual"].float()
            s["kept"].copy_(h)
            r["residual"] = s["kept"]
        x = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["weight"].float()
        if c["op"] == "norm":
            return dict(y=x.to(t), **r)
        x = _values(*_encode(x, c["kind"], c["row_group"]), c["row_group"])
    y = x @ _dense(s).t()
    if c["gated"]:
        gate, up = y.chunk(2, 1)
        y = gate / (1 + torch.exp(-gate)) * up
    return dict(y=y.to(t), **r)


def run(state: dict) -> dict:
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------ the definition in 64 bits
def _exact_code(y: torch.Tensor, kind: str, group: int) -> torch.Tensor:
    """What rows read back as: each part's largest magnitude spread over the code's range, to the nearest code."""
    top, out = CODE_MAX[kind], torch.empty_like(y)
    step = group or y.shape[1]
    for at in range(0, y.shape[1], step):
        part = y[:, at:at + step]
        scale = torch.clamp(part.abs().amax(1, keepdim=True) / top, min=SCALE_MIN)
        z = part / scale
        if kind == "int8":
            z = torch.round(z)
        else:  # three fraction bits down to an exponent of -6, below that steps of 2^-9
            unit = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)
            z = torch.round(z / unit) * unit
        out[:, at:at + step] = z.clamp(-top, top) * scale
    return out


def _exact_verify(s: dict) -> dict:
    c = s["c"]
    B, S = s["tokens"].shape
    picked, drafted = s["target"][:, :S].gather(2, s["tokens"][..., None])[..., 0].double().tolist(), None
    if c["draft"]:
        drafted = s["draft"].gather(2, s["tokens"][..., None])[..., 0].double().tolist()
    draws, last_draw, n, token = s["accept"].double().tolist(), s["final"].double(), s["counts"].tolist(), s["tokens"].tolist()
    out = torch.full((B, S + 1), -1, dtype=torch.int64)
    count = torch.zeros(B, dtype=torch.int32)
    for b in range(B):
        at = 0
        while at < n[b] and draws[b][at] * (drafted[b][at] if drafted else 1.0) < picked[b][at]:
            out[b, at] = token[b][at]
            at += 1
        mass = s["target"][b, at].double()
        if at < n[b]:
            less = mass.clone()
            if drafted:
                less -= s["draft"][b, at].double()
            else:
                less[token[b][at]] -= 1.0
            less[less < 0] = 0.0
            mass = less if bool((less > 0).any()) else mass
        sums = torch.cumsum(mass, 0)
        out[b, at] = int(torch.searchsorted(sums, last_draw[b] * sums[-1], right=True))
        count[b] = at
    return dict(tokens=out, accepted=count)


def exact(case: dict, seed: int):
    s = prepare(case, seed)
    c = s["c"]
    if c["op"] == "verify":
        return _exact_verify(s)
    r = {}
    if c["op"] == "product" and not c["kind"]:
        x = s["x"].double()
    elif c["op"] == "product":
        x = s["codes8"].double() * s["scale8"].double().repeat_interleave(c["row_group"] or c["k"], 1)
    else:
        h = s["x"].double()
        if c["residual"] != "none":
            h = r["residual"] = h + s["residual"].double()
        x = h / torch.sqrt((h ** 2).sum(1, keepdim=True) / c["k"] + EPS) * s["weight"].double()
        if c["op"] == "norm":
            return dict(y=x, **r)
        x = _exact_code(x, c["kind"], c["row_group"])
    y = torch.zeros(x.shape[0], c["n"], dtype=torch.float64, device=DEV)
    for i, at in enumerate(range(0, c["k"], c["group"])):  # a group of columns at a time
        end = min(at + c["group"], c["k"])
        columns = torch.arange(at, end, device=DEV)
        code = ((s["codes"][:, columns // 2] >> (4 * (columns % 2)).to(torch.uint8)) & 15).double()
        zero = s["zeros"][:, i:i + 1].double() if c["zeros"] else 8.0
        y += (x[:, at:end].contiguous() @ (code - zero).t().contiguous()) * s["scales"][:, i].double()
    if c["gated"]:
        half = c["n"] // 2
        y = y[:, :half] * torch.sigmoid(y[:, :half]) * y[:, half:]
    return dict(y=y, **r)
