"""Reference SOL of a decoder layer's ops, from the reference operators.

The analyzer's hotness weighs an op name by the gap between its SOL and a
reference, the SOL that the same op reaches elsewhere.  This module provides
that reference for the ops of a served model's attention layer, and with ``ffn``
for those of the whole decoder layer around it (norms, products with 4-bit
weights, verification of drafted tokens): it runs them
(``operators``) at given sizes, a prompt and then decode steps, records the
calls as a trace of CPU ops, launches and kernels with their operation counts
and logical bytes, and has the analyzer rate them (HERSCHEL_OUT_SOL).  An op's
time is the analyzer's, from its first kernel's start to its last one's end.

    python -m paper_2609_40247_amd.reference --prompt 4096 --batch 32 --cache fp8
    python -m paper_2609_40247_amd.reference --batch 4 --ffn 14336 --rows int8 --drafts 3 --vocab 151936

prints per op name the calls, the time of a call, MFU, MBU and SOL; the SOL column
is the ``ref_sol_ppm`` of traces of the same ops at the same sizes.
"""
from __future__ import annotations

import argparse
import bisect
import json
import os
import tempfile
from decimal import Decimal

import numpy as np
import torch
from torch.profiler import ProfilerActivity, profile, record_function

from . import herschel as H
from . import operators as O

CACHES = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn, "int8": torch.int8}
ROWS = {"16": None, "fp8": torch.float8_e4m3fn, "int8": torch.int8}
OPS = ("rope_write_prompt", "attn_prompt", "rope_write_step", "attn_decode")
PRODUCTS = ("qkv", "out", "gate", "down")
LAYER_OPS = tuple(f"{op}_{when}" for when in ("prompt", "step") for op in ("norm",) + tuple("product_" + p for p in PRODUCTS))
# MI355X: dense bf16 matrix rate and HBM3E bandwidth
PEAK_FLOPS, PEAK_BYTES = 2_500_000_000_000_000, 8_000_000_000_000


class AttentionLayer:
    """Rotary positions, cache and attention of one layer, for ``batch`` sequences of up to ``room`` tokens.

    ``prompt`` takes the QKV product's rows of whole prompts, ``step`` those of one new token a sequence; both
    return the attention's output rows.  Pages are given out in a fixed shuffled order.  A prompt longer than ``room``
    is refused; a step's token beyond it is not cached and its output no number, which ``cache.check`` reports."""

    def __init__(self, heads: int = 32, kv_heads: int = 8, head_dim: int = 128, batch: int = 1, room: int = 8192,
                 page_size: int = 64, cache="bf16", dtype=torch.bfloat16, stretch: float = 1.0, device="cuda", seed: int = 0,
                 new_tokens: int = 1):
        self.new_tokens = new_tokens
        self.heads, self.kv_heads, self.head_dim, self.batch, self.page_size = heads, kv_heads, head_dim, batch, page_size
        self.room = room
        pages = -(-room // page_size)
        self.cache = O.PagedCache.allocate(batch * pages, kv_heads, page_size, head_dim,
                                           CACHES[cache] if isinstance(cache, str) else cache, device)
        order = torch.randperm(batch * pages, generator=torch.Generator().manual_seed(seed))
        self.block_table = order.view(batch, pages).to(torch.int32).to(device)
        self.table = O.rotary_table(room, head_dim, stretch=stretch, device=device)
        self.lengths = torch.zeros(batch, dtype=torch.int32, device=device)
        self.decode = O.DecodeAttention(self.cache, batch=batch, heads=heads, new_tokens=new_tokens, dtype=dtype)

    def _split(self, qkv: torch.Tensor):
        h, g = self.heads, self.kv_heads
        return qkv[:, :h], qkv[:, h:h + g], qkv[:, h + g:]

    def _slots(self, seq: torch.Tensor, pos: torch.Tensor) -> torch.Tensor:
        pages = self.block_table.shape[1]
        slots = self.block_table[seq, (pos // self.page_size).clamp(0, pages - 1)].long() * self.page_size + pos % self.page_size
        # beyond a sequence's pages: beyond the cache, which the write reports
        return torch.where((pos >= 0) & (pos < pages * self.page_size), slots, self.block_table.numel() * self.page_size)

    def prompt(self, qkv: torch.Tensor, lengths: list, timed=lambda name, call: call()) -> torch.Tensor:
        """qkv [sum of lengths, heads + 2 kv heads, dim]: all sequences' prompts, one after the other."""
        dev = qkv.device
        if len(lengths) != self.batch or sum(lengths) != qkv.shape[0] or not all(0 <= n <= self.room for n in lengths):
            raise ValueError(f"lengths must be {self.batch} of at most {self.room} tokens, qkv's rows in all")
        n = torch.tensor(lengths, device=dev)
        seq = torch.repeat_interleave(torch.arange(self.batch, device=dev), n)
        cu = torch.cat([n.new_zeros(1), n.cumsum(0)])
        pos = torch.arange(qkv.shape[0], device=dev) - cu[seq]
        slots, cu = self._slots(seq, pos), cu.to(torch.int32)
        q, k, v = self._split(qkv)
        q, k = timed("rope_write_prompt", lambda: O.rope_write(q, k, v, pos, self.table, self.cache, slots, keep_keys=True))
        self.lengths.copy_(n)
        return timed("attn_prompt", lambda: O.attn_prompt(q, k, v, cu, max_q=max(lengths)))

    def step(self, qkv: torch.Tensor, timed=lambda name, call: call()) -> torch.Tensor:
        """qkv [batch * new tokens, heads + 2 kv heads, dim]: every sequence's next tokens, one after the other."""
        pos = (self.lengths.long()[:, None] + torch.arange(self.new_tokens, device=qkv.device)).view(-1)
        slots = self._slots(torch.arange(self.batch, device=qkv.device).repeat_interleave(self.new_tokens), pos)
        self.lengths += self.new_tokens
        q, k, v = self._split(qkv)
        q, _ = timed("rope_write_step", lambda: O.rope_write(q, k, v, pos, self.table, self.cache, slots))
        q = q.view(self.batch, self.new_tokens, *q.shape[1:])
        return timed("attn_decode", lambda: self.decode(q, self.block_table, self.lengths)).flatten(0, 1)


class DecoderLayer(AttentionLayer):
    """The attention layer with the norms and products around it: 4-bit weights [``group`` columns a scale], a gated
    feed-forward part of ``ffn``, ``rows`` of 16 bits, fp8 or int8 into the products behind the norms.

    ``prompt`` and ``step`` take rows of the block before and the residual stream [tokens, hidden], float32 or the
    rows' type, which they add to in place, and return the block's rows.  With ``new_tokens`` a step has a token
    and its drafts; ``keep`` takes back those that the verification did not accept.  Weights are random."""

    def __init__(self, *args, ffn: int = 14_336, rows="16", group: int = 128, zeros: bool = False, eps: float = 1e-6, **kw):
        super().__init__(*args, **kw)
        h, g, d = self.heads, self.kv_heads, self.head_dim
        self.hidden, self.ffn, self.eps = h * d, ffn, eps
        self.rows = ROWS[rows] if isinstance(rows, str) else rows
        dev = self.lengths.device
        draw = torch.Generator(device=dev).manual_seed(kw.get("seed", 0) + 1)

        def weights(n, k):
            return O.Weights4.quantise(torch.randn(n, k, generator=draw, device=dev) * k ** -0.5, group, zeros=zeros,
                                       scale_dtype=self.decode.dtype)
        self.weights = dict(qkv=weights((h + 2 * g) * d, self.hidden), out=weights(self.hidden, h * d),
                            gate=weights(2 * ffn, self.hidden), down=weights(self.hidden, ffn))
        self.norms = [(1 + 0.1 * torch.randn(self.hidden, generator=draw, device=dev)).to(self.decode.dtype) for _ in range(2)]

    def _block(self, x, residual, when: str, attend, timed):
        def norm(x, i):
            return timed("norm_" + when, lambda: O.norm_rows(x, self.norms[i], residual, eps=self.eps, kind=self.rows))

        def product(x, name, gated=False):
            return timed(f"product_{name}_{when}",
                         lambda: O.product4(x, self.weights[name], gated=gated, dtype=self.decode.dtype))
        o = attend(product(norm(x, 0), "qkv").view(x.shape[0], -1, self.head_dim))
        x = product(o.reshape(x.shape[0], -1), "out")
        return product(product(norm(x, 1), "gate", True), "down")

    def prompt(self, x: torch.Tensor, residual: torch.Tensor, lengths: list, timed=lambda name, call: call()) -> torch.Tensor:
        return self._block(x, residual, "prompt", lambda qkv: super(DecoderLayer, self).prompt(qkv, lengths, timed), timed)

    def step(self, x: torch.Tensor, residual: torch.Tensor, timed=lambda name, call: call()) -> torch.Tensor:
        return self._block(x, residual, "step", lambda qkv: super(DecoderLayer, self).step(qkv, timed), timed)

    def keep(self, accepted: torch.Tensor) -> None:
        """After a step of a token and its drafts: the cache holds the token and the accepted ones."""
        self.lengths -= self.new_tokens - 1 - accepted


def counts(layer: AttentionLayer, op: str, lengths: list, vocab: int = 0) -> tuple:
    """(operations, logical bytes) of a call over sequences of these lengths (for a step: with the new tokens):
    what it cannot do without, each input read once and each output written once."""
    h, g, d, e, new = layer.heads, layer.kv_heads, layer.head_dim, 2, getattr(layer, "new_tokens", 1)
    row = d * layer.cache.k.element_size() + (4 if layer.cache.quantised else 0)
    t = sum(lengths) if op.endswith("prompt") else len(lengths) * new
    if op.startswith("rope_write"):
        kept = t * g * d * e if op == "rope_write_prompt" else 0
        return 3 * t * (h + g) * d, t * ((2 * h + 2 * g) * d * e + 2 * g * row + 4 * d + 16) + kept
    if op == "attn_prompt":
        return sum(2 * d * h * n * (n + 1) for n in lengths), sum(lengths) * (2 * h + 2 * g) * d * e
    if op == "attn_decode":
        seen = sum(n - i for n in lengths for i in range(new))
        return 4 * d * h * seen, 2 * t * h * d * e + 2 * sum(lengths) * g * row
    if op == "verify_drafts":  # the row that a sequence's token is drawn from, of both models
        return 3 * len(lengths) * vocab, len(lengths) * (2 * vocab * 4 + (new - 1) * (16 + 8 + 8) + 16)
    to8 = layer.rows is not None
    if op.startswith("norm"):
        return 6 * t * layer.hidden, t * layer.hidden * (e + 2 * 4 + (1 if to8 else e)) + layer.hidden * e + (4 * t if to8 else 0)
    name = op.split("_")[1]
    w = layer.weights[name]
    x = t * w.k + 4 * t if to8 and name in ("qkv", "gate") else t * w.k * e  # the others' rows come with 16 bits
    return 2 * t * w.n * w.k, w.n * ((w.k + 1) // 2) + 4 * w.n * w.groups + x + t * (w.n // 2 if name == "gate" else w.n) * e


class Recorder:
    """Records calls as a trace, from torch's profiler: each call a CPU op, its launches and its kernels with the times
    that the device reports for them.  (Between events around a call there would be the host's time too.)"""

    def __init__(self, ops: tuple = OPS):
        self.ops = ops

    def begin(self) -> None:
        torch.cuda.synchronize()
        self.profile = profile(activities=[ProfilerActivity.CPU, ProfilerActivity.CUDA], acc_events=True)
        self.profile.start()

    def __call__(self, name: str, call):
        with record_function(name):
            return call()

    def columns(self, work: list) -> dict:
        """The trace's columns; ``work``: (operations, bytes) of each call in order.  ``kernels`` holds their names."""
        torch.cuda.synchronize()
        self.profile.stop()
        with tempfile.TemporaryDirectory() as folder:
            path = os.path.join(folder, "trace.json")
            self.profile.export_chrome_trace(path)
            with open(path) as f:
                events = [e for e in json.load(f, parse_float=Decimal)["traceEvents"] if e.get("ph") == "X"]

        def span(e):  # microseconds with three decimals: ns
            begin = int(Decimal(e["ts"]) * 1000)
            return begin, begin + max(1, int(Decimal(e["dur"]) * 1000))
        ops = sorted((e for e in events if e.get("cat") == "user_annotation" and e["name"] in self.ops), key=span)
        launches = {e["args"].get("correlation"): e for e in events if e.get("cat") == "cuda_runtime"}
        kernels = sorted((e for e in events if e.get("cat") == "kernel"), key=span)
        if len(ops) != len(work) or not kernels:
            raise RuntimeError(f"the profiler recorded {len(ops)} of {len(work)} calls and {len(kernels)} kernels")
        base = span(ops[0])[0]
        c = {k: [] for k in ("ts", "te", "corr", "pid", "lane", "name", "kind", "flops", "bytes")}
        self.kernels = []

        def row(kind, e, corr, name, f=0, b=0):
            begin, end = span(e)
            for k, x in zip(c, (begin - base, end - base, corr, 0, 0, name, kind, f, b)):
                c[k].append(x)
        for op, (f, b) in zip(ops, work):
            row(H.CPU_OP, op, 0, self.ops.index(op["name"]), f, b)
        begins = [span(op)[0] for op in ops]
        for i, kernel in enumerate(kernels):
            launch = launches.get(kernel["args"].get("correlation"))
            if launch is None:
                continue
            at = bisect.bisect_right(begins, span(launch)[0]) - 1
            if at < 0 or span(launch)[1] > span(ops[at])[1]:
                continue  # of no recorded call
            if kernel["name"] not in self.kernels:
                self.kernels.append(kernel["name"])
            row(H.LAUNCH, launch, i, 0)
            row(H.KERNEL, kernel, i, self.kernels.index(kernel["name"]))
        types = dict(ts=np.int64, te=np.int64, corr=np.int64, pid=np.int32, lane=np.int32, name=np.int32,
                     kind=np.uint8, flops=np.int64, bytes=np.int64)
        return {k: np.array(v, dtype=types[k]) for k, v in c.items()}


def _order(names: tuple, when: str) -> list:
    """The ops of a prompt or a step in the order of their calls."""
    mine = list(OPS[:2] if when == "prompt" else OPS[2:])
    if LAYER_OPS[0] in names:
        norm, (qkv, *others) = "norm_" + when, [f"product_{p}_{when}" for p in PRODUCTS]
        mine = [norm, qkv] + mine + [others[0], norm] + others[1:]
    return mine + (["verify_drafts"] if when == "step" and "verify_drafts" in names else [])


def reference_sol(heads: int = 32, kv_heads: int = 8, head_dim: int = 128, prompt: int = 4096, batch: int = 32,
                  prompts: int = 1, steps: int = 16, cache: str = "fp8", page_size: int = 64,
                  peak_flops: int = PEAK_FLOPS, peak_bytes: int = PEAK_BYTES, variant: str | None = None, ffn: int = 0,
                  rows: str = "16", drafts: int = 0, vocab: int = 32_000) -> dict:
    """Runs prompts of ``prompt`` tokens, ``prompts`` sequences a call, then ``steps`` decode steps of ``batch``
    sequences behind prompts of that length; with ``ffn`` the whole decoder layer, with ``drafts`` so many drafted
    tokens a sequence and step and their verification over ``vocab`` tokens.  Returns per op name the analyzer's
    calls, time (ns a call), MFU and MBU and SOL in parts per million, and the trace it rated (``columns``,
    ``params``)."""
    g = torch.Generator(device="cuda").manual_seed(0)
    new = drafts + 1
    names = OPS + (LAYER_OPS if ffn else ()) + (("verify_drafts",) if drafts else ())

    def layer(n, room, new_tokens):
        if ffn:
            return DecoderLayer(heads, kv_heads, head_dim, n, room, page_size, cache, ffn=ffn, rows=rows, new_tokens=new_tokens)
        return AttentionLayer(heads, kv_heads, head_dim, n, room, page_size, cache, new_tokens=new_tokens)

    def inputs(n):  # the QKV product's rows, or the block before's and the residual stream
        if not ffn:
            return (torch.randn(n, heads + 2 * kv_heads, head_dim, generator=g, device="cuda").to(torch.bfloat16),)
        return (torch.randn(n, heads * head_dim, generator=g, device="cuda").to(torch.bfloat16),
                torch.randn(n, heads * head_dim, generator=g, device="cuda"))
    first, then = layer(prompts, prompt, 1), layer(batch, prompt + (steps + 2) * new, new)
    given, lengths = inputs(prompts * prompt), [prompt] * prompts
    for b in range(batch):  # fill the decode layer's cache, a sequence at a time
        pos = torch.arange(prompt, device="cuda")
        qkv = torch.randn(prompt, heads + 2 * kv_heads, head_dim, generator=g, device="cuda").to(torch.bfloat16)
        q, k, v = then._split(qkv)
        O.rope_write(None, k, v, pos, then.table, then.cache, then._slots(torch.full_like(pos, b), pos))
    then.lengths.fill_(prompt)
    tokens = [inputs(batch * new) for _ in range(steps + 2)]
    if drafts:
        target = torch.softmax(3 * torch.randn(batch, new, vocab, generator=g, device="cuda"), -1)
        draft = torch.softmax(target[:, :-1].log() + 0.5 * torch.randn(batch, drafts, vocab, generator=g, device="cuda"), -1)
        drafted = torch.multinomial(draft.view(-1, vocab), 1, generator=g).view(batch, drafts)
        accept, final = (torch.rand(n, generator=g, device="cuda") for n in ((batch, drafts), (batch,)))

    def step(timed=lambda name, call: call()):
        then.step(*tokens.pop(), timed=timed)
        if drafts:
            timed("verify_drafts", lambda: O.verify_drafts(target, drafted, accept, final, draft=draft))
    rec, work = Recorder(names), []
    order = {when: _order(names, when) for when in ("prompt", "step")}
    for warm in range(2):  # once without and once under the profiler, whose first records take longer
        if warm:
            rec.begin()
        first.prompt(*given, lengths)
        step()
    for _ in range(max(1, steps // 4)):
        first.prompt(*given, lengths, timed=rec)
        work += [counts(first, op, lengths) for op in order["prompt"]]
    for i in range(steps):
        step(rec)
        work += [counts(then, op, [prompt + (3 + i) * new] * batch, vocab) for op in order["step"]]
    columns = rec.columns(work)
    first.cache.check()
    then.cache.check()
    params = dict(window_begin=int(columns["ts"].min()), window_end=int(columns["te"].max()) + 1, gap_threshold=0,
                  n_procs=1, n_streams=1, n_threads=1, n_names=max(1, len(rec.kernels)), n_op_names=len(names),
                  flags=H.OUT_CONTAIN | H.OUT_SOL, peak_flops=peak_flops, peak_bytes=peak_bytes)
    code, out = H.analyze(columns, params, variant=variant)
    if code != H.OK:
        raise RuntimeError(f"analyze: {H.herschel_strerror(code)}")
    ops = {}
    for i, name in enumerate(names):
        mine = (columns["kind"] == H.CPU_OP) & (columns["name"] == i) & (out["op_sol"] >= 0)
        t, f, b = int(out["opn_time"][i]), int(out["opn_flops"][i]), int(out["opn_bytes"][i])
        ops[name] = dict(calls=int(mine.sum()), ns=t // max(1, int(mine.sum())), mfu=f * 10 ** 15 // max(1, t * peak_flops),
                         mbu=b * 10 ** 15 // max(1, t * peak_bytes), sol=int(out["opn_sol"][i]))
    return dict(ops=ops, columns=columns, params=params, outputs=out)


def main() -> None:
    ap = argparse.ArgumentParser(description="Reference SOL of a decoder layer's ops on this GPU.")
    for name, value in (("heads", 32), ("kv-heads", 8), ("head-dim", 128), ("prompt", 4096), ("prompts", 1), ("batch", 32),
                        ("steps", 16), ("page-size", 64), ("ffn", 0), ("drafts", 0), ("vocab", 32_000)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--cache", choices=sorted(CACHES), default="fp8")
    ap.add_argument("--rows", choices=sorted(ROWS), default="16", help="of the products behind the norms")
    a = vars(ap.parse_args())
    if a["cache"] == "f16":
        ap.error("the rows of this command are bf16: bf16, fp8 or int8")
    r = reference_sol(**a)
    print(f"{'op':<20}{'calls':>6}{'us':>10}{'MFU ppm':>10}{'MBU ppm':>10}{'SOL ppm':>10}")
    for name, o in r["ops"].items():
        print(f"{name:<20}{o['calls']:>6}{o['ns'] / 1000:>10.1f}{o['mfu']:>10}{o['mbu']:>10}{o['sol']:>10}")


if __name__ == "__main__":
    main()
