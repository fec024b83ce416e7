"""Reference SOL of an attention layer's ops, from the reference operators.

The analyzer's hotness weighs an op name by the gap between its SOL and a
reference, the SOL that the same op reaches elsewhere.  This module provides
that reference for the ops of a served model's attention layer: it runs them
(``operators``) at given sizes, a prompt and then decode steps, records the
calls as a trace of CPU ops, launches and kernels with their operation counts
and logical bytes, and has the analyzer rate them (HERSCHEL_OUT_SOL).  An op's
time is the analyzer's, from its first kernel's start to its last one's end.

    python -m paper_2609_40247_amd.reference --prompt 4096 --batch 32 --cache fp8

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
OPS = ("rope_write_prompt", "attn_prompt", "rope_write_step", "attn_decode")
# MI355X: dense bf16 matrix rate and HBM3E bandwidth
PEAK_FLOPS, PEAK_BYTES = 2_500_000_000_000_000, 8_000_000_000_000


class AttentionLayer:
    """Rotary positions, cache and attention of one layer, for ``batch`` sequences of up to ``room`` tokens.

    ``prompt`` takes the QKV product's rows of whole prompts, ``step`` those of one new token a sequence; both
    return the attention's output rows.  Pages are given out in a fixed shuffled order.  A prompt longer than ``room``
    is refused; a step's token beyond it is not cached and its output no number, which ``cache.check`` reports."""

    def __init__(self, heads: int = 32, kv_heads: int = 8, head_dim: int = 128, batch: int = 1, room: int = 8192,
                 page_size: int = 64, cache="bf16", dtype=torch.bfloat16, stretch: float = 1.0, device="cuda", seed: int = 0):
        self.heads, self.kv_heads, self.head_dim, self.batch, self.page_size = heads, kv_heads, head_dim, batch, page_size
        self.room = room
        pages = -(-room // page_size)
        self.cache = O.PagedCache.allocate(batch * pages, kv_heads, page_size, head_dim,
                                           CACHES[cache] if isinstance(cache, str) else cache, device)
        order = torch.randperm(batch * pages, generator=torch.Generator().manual_seed(seed))
        self.block_table = order.view(batch, pages).to(torch.int32).to(device)
        self.table = O.rotary_table(room, head_dim, stretch=stretch, device=device)
        self.lengths = torch.zeros(batch, dtype=torch.int32, device=device)
        self.decode = O.DecodeAttention(self.cache, batch=batch, heads=heads, dtype=dtype)

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
        """qkv [batch, heads + 2 kv heads, dim]: every sequence's next token."""
        pos = self.lengths.long()
        slots = self._slots(torch.arange(self.batch, device=qkv.device), pos)
        self.lengths += 1
        q, k, v = self._split(qkv)
        q, _ = timed("rope_write_step", lambda: O.rope_write(q, k, v, pos, self.table, self.cache, slots))
        return timed("attn_decode", lambda: self.decode(q[:, None], self.block_table, self.lengths))[:, 0]


def counts(layer: AttentionLayer, op: str, lengths: list) -> tuple:
    """(operations, logical bytes) of a call over sequences of these lengths (for a step: with the new token):
    what it cannot do without, each input read once and each output written once."""
    h, g, d, e = layer.heads, layer.kv_heads, layer.head_dim, 2
    row = d * layer.cache.k.element_size() + (4 if layer.cache.quantised else 0)
    if op.startswith("rope_write"):
        t = sum(lengths) if op == "rope_write_prompt" else len(lengths)
        kept = t * g * d * e if op == "rope_write_prompt" else 0
        return 3 * t * (h + g) * d, t * ((2 * h + 2 * g) * d * e + 2 * g * row + 4 * d + 16) + kept
    if op == "attn_prompt":
        return sum(2 * d * h * n * (n + 1) for n in lengths), sum(lengths) * (2 * h + 2 * g) * d * e
    return sum(4 * d * h * n for n in lengths), 2 * len(lengths) * h * d * e + 2 * sum(lengths) * g * row


class Recorder:
    """Records calls as a trace, from torch's profiler: each call a CPU op, its launches and its kernels with the times
    that the device reports for them.  (Between events around a call there would be the host's time too.)"""

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
        ops = sorted((e for e in events if e.get("cat") == "user_annotation" and e["name"] in OPS), key=span)
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
            row(H.CPU_OP, op, 0, OPS.index(op["name"]), f, b)
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


def reference_sol(heads: int = 32, kv_heads: int = 8, head_dim: int = 128, prompt: int = 4096, batch: int = 32,
                  prompts: int = 1, steps: int = 16, cache: str = "fp8", page_size: int = 64,
                  peak_flops: int = PEAK_FLOPS, peak_bytes: int = PEAK_BYTES, variant: str | None = None) -> dict:
    """Runs prompts of ``prompt`` tokens, ``prompts`` sequences a call, then ``steps`` decode steps of ``batch``
    sequences behind prompts of that length.  Returns per op name the analyzer's calls, time (ns a call), MFU and
    MBU and SOL in parts per million, and the trace it rated (``columns``, ``params``)."""
    g = torch.Generator(device="cuda").manual_seed(0)
    width = heads + 2 * kv_heads

    def qkv(n):
        return torch.randn(n, width, head_dim, generator=g, device="cuda").to(torch.bfloat16)
    first = AttentionLayer(heads, kv_heads, head_dim, prompts, prompt, page_size, cache)
    then = AttentionLayer(heads, kv_heads, head_dim, batch, prompt + steps + 2, page_size, cache)
    rows, lengths = qkv(prompts * prompt), [prompt] * prompts
    for b in range(batch):  # fill the decode layer's cache, a sequence at a time
        pos = torch.arange(prompt, device="cuda")
        q, k, v = then._split(qkv(prompt))
        O.rope_write(None, k, v, pos, then.table, then.cache, then._slots(torch.full_like(pos, b), pos))
    then.lengths.fill_(prompt)
    tokens = [qkv(batch) for _ in range(steps + 2)]
    rec, work = Recorder(), []
    for warm in range(2):  # once without and once under the profiler, whose first records take longer
        if warm:
            rec.begin()
        first.prompt(rows, lengths)
        then.step(tokens.pop())
    for _ in range(max(1, steps // 4)):
        first.prompt(rows, lengths, rec)
        work += [counts(first, op, lengths) for op in OPS[:2]]
    for i in range(steps):
        then.step(tokens.pop(), rec)
        work += [counts(then, op, [prompt + 3 + i] * batch) for op in OPS[2:]]
    columns = rec.columns(work)
    first.cache.check()
    then.cache.check()
    params = dict(window_begin=int(columns["ts"].min()), window_end=int(columns["te"].max()) + 1, gap_threshold=0,
                  n_procs=1, n_streams=1, n_threads=1, n_names=max(1, len(rec.kernels)), n_op_names=len(OPS),
                  flags=H.OUT_CONTAIN | H.OUT_SOL, peak_flops=peak_flops, peak_bytes=peak_bytes)
    code, out = H.analyze(columns, params, variant=variant)
    if code != H.OK:
        raise RuntimeError(f"analyze: {H.herschel_strerror(code)}")
    ops = {}
    for i, name in enumerate(OPS):
        mine = (columns["kind"] == H.CPU_OP) & (columns["name"] == i) & (out["op_sol"] >= 0)
        t, f, b = int(out["opn_time"][i]), int(out["opn_flops"][i]), int(out["opn_bytes"][i])
        ops[name] = dict(calls=int(mine.sum()), ns=t // max(1, int(mine.sum())), mfu=f * 10 ** 15 // max(1, t * peak_flops),
                         mbu=b * 10 ** 15 // max(1, t * peak_bytes), sol=int(out["opn_sol"][i]))
    return dict(ops=ops, columns=columns, params=params, outputs=out)


def main() -> None:
    ap = argparse.ArgumentParser(description="Reference SOL of an attention layer's ops on this GPU.")
    for name, value in (("heads", 32), ("kv-heads", 8), ("head-dim", 128), ("prompt", 4096), ("prompts", 1), ("batch", 32),
                        ("steps", 16), ("page-size", 64)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--cache", choices=sorted(CACHES), default="fp8")
    a = vars(ap.parse_args())
    if a["cache"] == "f16":
        ap.error("the rows of this command are bf16: bf16, fp8 or int8")
    r = reference_sol(**a)
    print(f"{'op':<20}{'calls':>6}{'us':>10}{'MFU ppm':>10}{'MBU ppm':>10}{'SOL ppm':>10}")
    for name, o in r["ops"].items():
        print(f"{name:<20}{o['calls']:>6}{o['ns'] / 1000:>10.1f}{o['mfu']:>10}{o['mbu']:>10}{o['sol']:>10}")


if __name__ == "__main__":
    main()
