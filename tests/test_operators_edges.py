"""The reference operators where their inputs are extreme.

Bounds are derived as in the operators' other tests.  For half rows one term
joins them.  The exponentials enter the second product as halves: above 2^-14
they are off by half a last place, below that by 2^-25 at most, where the row's
largest stands at 2^6 or above when it is met.  So a key loses at most 2^-31 of
the largest weight; and where a step's keys have so little that a lane's sum (of
8 to 32 keys) would be below 2^-12, the reference moves and puts the step's
largest at 2^-4: keys within 9 powers of two of it lose no more than half a last
place.
"""
from __future__ import annotations

import ctypes
import math
import time

import pytest
import torch

from paper_2609_40247_amd import herschel as H
from paper_2609_40247_amd import operators as O
from test_host_calls import child, fake, launches  # noqa: F401 (a fixture)
from test_operators import (BF, DEV, F8, HF, I8, U, check_attention, dense, exact_attention, fake_cache, fill_cache, gpu, lib,
                            make_cache, paged, rand, rope_args, run_decode, run_prompt)


# ------------------------------------------------------------ weights far below a row's largest
def sinking(nq, nk, hq, hk, D, at, gap, seed=0):
    """Half rows: key `at` has the largest score of every query and the value 0; the others' scores lie gap[0] to
    gap[1] below it (and a little noise), their values from 0.5 to 1.5."""
    q, k = rand(nq, hq, D, seed=seed, dtype=HF, gain=0.02), rand(nk, hk, D, seed=seed + 1, dtype=HF)
    u = torch.rand(nk, hk, generator=torch.Generator().manual_seed(seed + 2))
    q[:, :, 0] = 8
    k[:, :, 0] = (-(gap[0] + (gap[1] - gap[0]) * u) / 8).to(HF)
    v = (torch.rand(nk, hk, D, generator=torch.Generator().manual_seed(seed + 3)) + 0.5).to(HF)
    k[at, :, 0] = 0
    v[at] = 0
    return q, k, v


def check_sunk(out, lse, ref, n_keys, D, gap):
    """`check_attention` with the halves' further term; the values are at most 1.5."""
    # from 17 on a lane's 32 keys sum to less than 32 e^-17 2^6 = 2^-13.5: of all steps but the largest key's own (64 keys
    # at most) the reference moves, and the keys lie within 6 (8.7 powers of two) and the noise of each other
    lost = (64 if gap[0] > 17 else n_keys) * 2.0 ** -31 * 1.5
    o, l, A, S = ref
    d = (D + 8) * 2.0 ** -24 * S
    tol = (U[HF] * o.abs() + (1 + 2.0 ** -7) * ((U[HF] + 2 * d[..., None] + (n_keys + 16) * 2.0 ** -23) * A + lost) +
           2.0 ** -25)
    err = (out.double().cpu() - o).abs()
    assert (err <= tol).all(), (err.max(), tol[err == err.max()])
    if lse is not None:
        assert ((lse.double().cpu() - l).abs() <= d + (n_keys + 16) * 2.0 ** -23 + 2.0 ** -22 * l.abs()).all()


GAPS = [(17.4, 17.4), (10.0, 17.5), (24.0, 30.0)]
SINK_CASES = [  # queries, keys, heads, kv heads, D, rows of another sequence that sees no key, key with the largest score
    (20, 12_000, 4, 1, 64, 0, 0),           # parts of few rows
    (20, 12_000, 4, 2, 128, 0, 7000),
    (100, 2000, 2, 1, 128, 0, 0),           # few rows
    (100, 2000, 2, 1, 64, 0, 1999),
    (40, 3000, 4, 1, 128, 8000, 0),         # workgroups of 128 rows
    (40, 3000, 4, 2, 64, 12_000, 1500),
    (1400, 5000, 8, 2, 128, 0, 0),          # and in parts
]


@gpu
@pytest.mark.parametrize("gap", GAPS, ids=str)
@pytest.mark.parametrize("case", SINK_CASES, ids=str)
def test_weights_far_below_the_largest(case, gap):
    """One key takes nearly all the weight and has the value 0: the output is what thousands of small weights give."""
    nq, nk, hq, hk, D, more, at = case
    q, k, v = sinking(nq, nk, hq, hk, D, at, gap)
    rest = torch.zeros(more, hq, D, dtype=HF)
    cu_q, cu_k = (torch.tensor(c, dtype=torch.int32, device=DEV) for c in ([0, nq, nq + more], [0, nk, nk]))
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    n = 3 if more else 2
    out, lse = O.attn_prompt(torch.cat([q, rest]).to(DEV), k.to(DEV), v.to(DEV), cu_q[:n].contiguous(), cu_k[:n].contiguous(),
                             max_q=max(nq, more), scale=1.0, causal=False, return_lse=True, status=status)
    assert status.item() == 0
    rows = [r for r in (0, 1, 31, 32, 39, 99, 127, 128, 700, 1399) if r < nq]
    check_sunk(out[rows], lse[rows], exact_attention(q[rows], k, v, 1.0, False, 0), nk, D, gap)


@gpu
@pytest.mark.parametrize("gap", GAPS, ids=str)
def test_weights_far_below_the_largest_of_long_prompts(gap):
    """The same in workgroups of 256 rows; the largest score in the last tile of one sequence, in a middle one of the other."""
    n, m, hq, hk, D = 1024, [1500, 2100], 128, 2, 128
    parts = [sinking(n, x, hq, hk, D, at, gap, seed=10 * i) for i, (x, at) in enumerate(zip(m, (1499, 700)))]
    q, k, v = (torch.cat(t) for t in zip(*parts))
    cu_q, cu_k = (torch.tensor(c, dtype=torch.int32, device=DEV) for c in ([0, n, 2 * n], [0, m[0], sum(m)]))
    out, lse = O.attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), cu_q, cu_k, max_q=n, scale=1.0, causal=False, return_lse=True)
    for i, (x, (pq, pk, pv)) in enumerate(zip(m, parts)):
        for r in (0, 33, 255, 256, 1023):
            for h in (0, 63, 64, 127):
                ref = exact_attention(pq[r:r + 1, h:h + 1], pk[:, h // 64:h // 64 + 1], pv[:, h // 64:h // 64 + 1], 1.0, False, 0)
                check_sunk(out[i * n + r:i * n + r + 1, h:h + 1], lse[i * n + r:i * n + r + 1, h:h + 1], ref, x, D, gap)


@gpu
@pytest.mark.parametrize("gap", GAPS, ids=str)
@pytest.mark.parametrize("lens,hq,hk,D,new,at", [([12_000], 4, 1, 64, 1, 0), ([3000, 700], 4, 2, 128, 1, 600),
                                                 ([131_000], 2, 2, 64, 1, 5), ([5000, 200], 20, 1, 128, 2, 3)], ids=str)
def test_decode_weights_far_below_the_largest(lens, hq, hk, D, new, at, gap):
    page = 64
    c = make_cache(HF, sum(-(-n // page) for n in lens) + 1, hk, page, D)
    bt = paged(c, lens, 3)
    q = torch.empty(len(lens), new, hq, D, dtype=HF)
    for b, n in enumerate(lens):
        q[b], k, v = sinking(new, n, hq, hk, D, at, gap, seed=10 * b)
        ids = bt[b, :-(-n // page)].long()
        for t, x in ((c.k, k), (c.v, v)):
            whole = torch.zeros(len(ids) * page, hk, D, dtype=HF)
            whole[:n] = x
            t[ids.to(DEV)] = whole.view(len(ids), page, hk, D).transpose(1, 2).contiguous().to(DEV)
    dec = O.DecodeAttention(c, batch=len(lens), heads=hq, new_tokens=new, dtype=HF)
    out, lse = dec(q.to(DEV), bt.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), scale=1.0, return_lse=True)
    c.check()
    for b, (k, v) in enumerate(dense(c, bt, lens)):
        check_sunk(out[b], lse[b], exact_attention(q[b], k, v, 1.0, True, 0), lens[b], D, gap)


@gpu
@pytest.mark.parametrize("gap", GAPS, ids=str)
@pytest.mark.parametrize("D", [64, 128])
def test_decode_weights_far_below_the_largest_of_long_shares(D, gap):
    """So many sequences and heads that a workgroup goes through most of a sequence; all of them share one's pages."""
    n, page, heads, B = 3000, 256, 32, 16
    c = make_cache(HF, -(-n // page), heads, page, D)
    q, k, v = sinking(1, n, heads, heads, D, 1, gap)
    for t, x in ((c.k, k), (c.v, v)):
        whole = torch.zeros(c.n_pages * page, heads, D, dtype=HF)
        whole[:n] = x
        t.copy_(whole.view(c.n_pages, page, heads, D).transpose(1, 2))
    bt = torch.arange(c.n_pages, dtype=torch.int32, device=DEV).repeat(B, 1)
    dec = O.DecodeAttention(c, batch=B, heads=heads, dtype=HF)
    out = dec(q.expand(B, 1, heads, D).contiguous().to(DEV), bt, torch.full((B,), n, dtype=torch.int32, device=DEV), scale=1.0)
    ref = exact_attention(q, k, v, 1.0, True, 0)
    for b in range(B):
        check_sunk(out[b], None, ref, n, D, gap)


# ------------------------------------------------------------ values that are not finite
@gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
@pytest.mark.parametrize("lens,D,window", [([37, 64, 129, 1], 128, 0), ([160, 33, 31], 64, 0), ([200, 97], 128, 50),
                                           ([300, 4000], 64, 64)], ids=str)
def test_decode_infinite_values_of_seen_keys(lens, D, window, dtype):
    """One new token: infinities in the last key's value and in the first one's that is seen stay infinities, at lengths
    that end inside a step and at its end."""
    page = 16

    def edit(c, bt):
        for b, n in enumerate(lens):
            first = max(0, n - window) if window else 0
            for key, head, d, x in ((n - 1, 0, 3, math.inf), (n - 1, 1, 4, -math.inf), (first, 0, 5, -math.inf),
                                    (first, 1, 6, math.inf), (n - 1, 1, 7, math.nan)):
                c.v[int(bt[b, key // page]), head, key % page, d] = x
    run_decode(lens, 4, 2, D, dtype, dtype, page, window=window, edit=edit)


@gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
@pytest.mark.parametrize("D,new", [(64, 1), (128, 1), (64, 2)])
def test_decode_infinite_values_of_small_weights(D, new, dtype):
    """A key hundreds below the largest score, with an infinite value: its weight is no longer a 32-bit number, but not 0."""
    lens, page, heads = [300, 64], 32, 2

    def edit(c, bt):
        q = rand(len(lens), new, heads, D, seed=2, dtype=dtype)  # the call's own rows
        for b, n in enumerate(lens):
            for h in range(heads):
                for key in (20, n - 30):
                    at = int(bt[b, key // page]), h, key % page
                    c.k[at] = (-16 * q[b].float().sum(0)[h] * (1.0 if new == 1 else 0.5)).to(dtype).to(DEV)
                    c.v[at][5] = math.inf
    run_decode(lens, heads, heads, D, dtype, dtype, page, new=new, edit=edit)


# ------------------------------------------------------------ huge values
@gpu
@pytest.mark.parametrize("low", [32, 128, 1024])
@pytest.mark.parametrize("D", [64, 128])
def test_decode_huge_values_of_small_weights(D, low):
    """The first keys lie hundreds below the others' scores and have values of 1e36: nothing of them is left, whether the
    higher scores come in the same wave, in another one or in another workgroup."""
    lens, page, heads = [4000, low + 1, low + 40], 16, 2

    def edit(c, bt):
        q = rand(len(lens), 1, heads, D, seed=2)
        for b in range(len(lens)):
            for key in range(low):
                at = int(bt[b, key // page]), slice(None), key % page
                c.k[at] = (-16 * q[b, 0]).to(DEV)
                c.v[at] = 1e36
    run_decode(lens, heads, heads, D, BF, BF, page, edit=edit)


@gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("more", [0, 16_000])
def test_prompt_huge_values_of_small_weights(D, more):
    """The same of prompts, also in rows that see a NaN in another dimension."""
    for bad in (False, True):
        def edit(q, k, v):
            q[:, :, 0] = 16
            k[:, :, 0] = 0
            k[:70, :, 0] = -16.0 * D ** 0.5
            v[:70] = 1e36
            if bad:
                v[100, :, 5] = math.nan
        run_prompt([40, more], [150, 0], 2, 1, D, BF, False, 0, edit=edit)


@gpu
@pytest.mark.parametrize("D", [64, 128])
def test_largest_values(D):
    """Values of 3e38 under equal scores: their mean is a number, though their sum is none."""
    for bad in (False, True):
        def edit(q, k, v):
            q *= 0
            v[:] = 3e38
            v[:, :, 1] = -3e38
            if bad:
                v[7, :, 5] = math.nan
        run_prompt([40], [3000], 2, 1, D, BF, False, 0, edit=edit)            # parts of few rows
        run_prompt([40, 16_000], [1000, 0], 2, 1, D, BF, False, 0, edit=edit)

    def fill(c, bt):
        c.k.zero_()
        c.v.fill_(3e38)
    run_decode([3000, 33], 4, 2, D, BF, BF, 16, edit=fill)


# ------------------------------------------------------------ rows without a query
NO_QUERY_CASES = [  # queries, rows before, rows after, heads, kv heads, D, keys beyond the queries
    ([5, 40, 1], 0, 17, 4, 2, 64, 0),                        # few rows
    ([1, 300] + [1, 2] * 15, 0, 9, 8, 2, 64, 0),             # packed
    ([1, 300] + [1, 2] * 15, 3, 0, 4, 4, 128, 0),
    ([0, 0], 0, 33, 4, 2, 128, 0),                           # padding alone
    ([30], 0, 3, 8, 2, 128, 4000),                           # parts of few rows
    ([700, 300], 0, 200, 20, 4, 128, 0),                     # workgroups of 128 rows
    ([900, 0, 500], 4, 200, 16, 16, 64, 0),
    ([1400], 0, 10, 8, 2, 128, 4000),                        # and in parts
    ([1030, 1026], 0, 300, 64, 16, 128, 0),                  # of 256 rows
]


@gpu
@pytest.mark.parametrize("case", NO_QUERY_CASES, ids=lambda c: f"{len(c[0])}-{sum(c[0])}-{c[1]}-{c[2]}-{c[5]}")
def test_prompt_rows_without_a_query(case):
    """Rows before the first sequence, after the last and beyond max_q are 0 with a log sum of minus infinity; the others
    are as without them."""
    nq, before, after, hq, hk, D, more = case
    n, nk = sum(nq), [x + more for x in nq]
    q, k, v = rand(n, hq, D, seed=1), rand(sum(nk), hk, D, seed=2), rand(sum(nk), hk, D, seed=3)
    padded = torch.cat([rand(before, hq, D, seed=4), q, rand(after, hq, D, seed=5)]).to(DEV)
    k, v, q = k.to(DEV), v.to(DEV), q.to(DEV)
    cu_q, cu_k = (torch.tensor([0] + x).cumsum(0).int().to(DEV) for x in (nq, nk))
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for most in (max(nq), max(nq) // 2):
        out = torch.full_like(padded, math.nan)
        status.zero_()
        got, lse = O.attn_prompt(padded, k, v, cu_q + before, cu_k, max_q=most, return_lse=True, out=out, status=status)
        assert got is out and status.item() == (O.BAD_LENGTH if before or most < max(nq) else 0)
        want, want_lse = O.attn_prompt(q, k, v, cu_q, cu_k, max_q=max(nq), return_lse=True)
        named = torch.zeros(before + n + after, dtype=torch.bool, device=DEV)
        named[before:before + n] = torch.cat([torch.arange(x, device=DEV) < most for x in nq])
        assert (out[~named] == 0).all() and (lse[~named] == -math.inf).all()
        rows = named[before:before + n]
        # another grid may add parts in another order
        assert torch.allclose(out[named].float(), want[rows].float(), rtol=2 ** -7, atol=2 ** -9)
        assert torch.allclose(lse[named], want_lse[rows], rtol=1e-5, atol=1e-5)


@gpu
def test_prompt_starts_that_fall_leave_no_row_unwritten():
    q = rand(300, 4, 64).to(DEV)
    k = rand(300, 2, 64, seed=1).to(DEV)
    for heads in (4, 1):
        for cu in ([5, 0, 10, 200], [0, 200, 50, 60], [40, 90, 20, 20], [-3, 10, 5, 290], [300, 300, 300, 300], [7, 7, 7, 7]):
            cu = torch.tensor(cu, dtype=torch.int32, device=DEV)
            for n in (1, 40):  # with empty ones that make the call a packed one
                starts = torch.cat([cu, cu[-1:].repeat(n)])
                status = torch.zeros(1, dtype=torch.int32, device=DEV)
                x = q[:, :heads]
                out = torch.full(x.shape, math.nan, dtype=BF, device=DEV)
                kv = k if heads == 4 else k[:, :1]
                O.attn_prompt(x, kv, kv, starts, starts.clamp(0, 300), max_q=300, out=out, status=status)
                assert status.item() == O.BAD_LENGTH and torch.isfinite(out).all(), (heads, cu.tolist(), n)


# ------------------------------------------------------------ empty calls
def test_rotary_write_of_no_tokens_needs_no_addresses():
    """Empty tensors have the address 0."""
    none = dict(q=None, k=None, v=None, q_out=None, positions=None, slots=None, n_tokens=0)
    L = lib()
    assert L.herschel_rope_write(ctypes.byref(rope_args(**none)), ctypes.byref(fake_cache())) == H.OK
    assert L.herschel_rope_write(ctypes.byref(rope_args(**none)), None) == H.OK
    for bad in (dict(head_dim=63), dict(rotary_dim=66), dict(layout=2), dict(type=O.FP8), dict(q_strides=O._Strides(-1, 64))):
        assert L.herschel_rope_write(ctypes.byref(rope_args(**{**none, **bad})), None) == H.EINVAL
    assert L.herschel_rope_write(ctypes.byref(rope_args(**none)), ctypes.byref(fake_cache(n_pages=0))) == H.EINVAL


@gpu
@pytest.mark.parametrize("kind", [None, BF, F8], ids=str)
def test_rotary_write_of_no_tokens(kind):
    x = torch.empty(0, 8, 64, dtype=BF, device=DEV)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    table = O.rotary_table(10, 64, device=DEV)
    cache = make_cache(kind, 2, 2, 16, 64, fill=0x11) if kind else None
    q, k = O.rope_write(x[:, :4], x[:, 4:6], x[:, 6:], none, table, cache, none if kind else None, keep_keys=True)
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)
    if cache:
        cache.check()
        assert (cache.k.view(torch.uint8) == 0x11).all()


@gpu
def test_decode_of_no_sequences():
    c = make_cache(BF, 2, 2, 16, 64)
    dec = O.DecodeAttention(c, batch=3, heads=4, new_tokens=2)
    none = torch.empty(0, 4, dtype=torch.int32, device=DEV)
    out, lse = dec(torch.empty(0, 2, 4, 64, dtype=BF, device=DEV), none, none[:, 0].contiguous(), return_lse=True)
    assert out.shape == (0, 2, 4, 64) and lse.shape == (0, 2, 4) and out.dtype == BF
    with pytest.raises(ValueError):
        dec(torch.empty(0, 2, 3, 64, dtype=BF, device=DEV), none, none[:, 0].contiguous())


# ------------------------------------------------------------ the recorded trace
@gpu
def test_recorded_kernels_have_their_own_times():
    """A call that keeps the host busy before and between its launches takes no longer on the device: a trace's kernels
    are the kernels, each with its launch inside its op."""
    from paper_2609_40247_amd import reference as R
    layer = R.AttentionLayer(8, 2, 64, 3, 400, 32, "fp8")
    qkv = rand(3, 12, 64).to(DEV)
    layer.lengths.fill_(300)
    layer.step(qkv)
    rec = R.Recorder()
    rec.begin()

    def slow(name, call):
        def late():
            time.sleep(0.003)
            return call()
        return rec(name, late)
    for _ in range(3):
        layer.step(qkv, slow)
    c = rec.columns([(1, 1)] * 6)
    ops, kernels, launches = (c["kind"] == x for x in (R.H.CPU_OP, R.H.KERNEL, R.H.LAUNCH))
    assert [R.OPS[i] for i in c["name"][ops]] == ["rope_write_step", "attn_decode"] * 3
    assert kernels.sum() == launches.sum() == 9  # one of a write, two of an attention
    names = [rec.kernels[i] for i in c["name"][kernels]]
    assert ["k_rope" in n for n in names] == [True, False, False] * 3 and sum("k_decode_join" in n for n in names) == 3
    spans = list(zip(c["ts"], c["te"]))
    host, device = [s for s, x in zip(spans, ops) if x], [s for s, x in zip(spans, kernels) if x]
    assert all(b - a > 3_000_000 for a, b in host) and all(0 < b - a < 1_000_000 for a, b in device)
    for i, (a, b) in enumerate(s for s, x in zip(spans, launches) if x):
        op = host[2 * (i // 3) + (i % 3 > 0)]
        assert op[0] <= a and b <= op[1] and device[i][0] >= a


# ------------------------------------------------------------ a layer's room
def test_layer_refuses_prompts_beyond_its_room():
    """What would index the block table beyond its end, which on a GPU ends the process, is refused or kept inside."""
    from paper_2609_40247_amd import reference as R
    layer = R.AttentionLayer.__new__(R.AttentionLayer)
    layer.batch, layer.room, layer.page_size = 2, 40, 16
    layer.block_table = torch.tensor([[4, 1, 0], [2, 5, 3]], dtype=torch.int32)
    x = torch.zeros(50, 6, 64)
    for lengths in ([41, 9], [50], [25, 24], [25, 26], [51, -1], [10, 20, 20]):
        with pytest.raises(ValueError, match="lengths"):
            layer.prompt(x, lengths)
    seq, pos = torch.tensor([0, 0, 1, 1, 0, 1]), torch.tensor([0, 47, 16, 48, 1 << 40, -1])
    assert layer._slots(seq, pos).tolist() == [64, 15, 80, 96, 96, 96]  # 96: beyond the cache


@gpu
def test_layer_reports_steps_beyond_its_room():
    from paper_2609_40247_amd import reference as R
    layer = R.AttentionLayer(4, 2, 64, 2, 32, 16, "bf16")
    x = rand(62, 8, 64).to(DEV)
    layer.prompt(x, [31, 31])
    layer.step(x[:2])
    layer.cache.check()
    before = layer.cache.k.clone(), layer.cache.v.clone()
    for _ in range(20):  # across the last page's end
        layer.step(x[:2])
        with pytest.raises(ValueError, match="position"):
            layer.cache.check()
    assert torch.equal(layer.cache.k, before[0]) and torch.equal(layer.cache.v, before[1])


# ------------------------------------------------------------ graphs of one handle
class Seen:
    """The library, with the workspaces that decode calls were given."""

    def __init__(self):
        self.lib, self.workspaces = lib(), []
        self.herschel_attn_decode_workspace = self.lib.herschel_attn_decode_workspace

    def herschel_attn_decode(self, args, cache):
        fields = [f for f, _ in O.HerschelDecodeArgs._fields_]
        flat = O._DECODE.unpack(args)  # q_strides are two values
        self.workspaces.append(flat[fields.index("workspace") + 1])
        return self.lib.herschel_attn_decode(args, cache)


@gpu
def test_graphs_of_one_handle_have_workspaces_of_their_own():
    seen = Seen()
    c = make_cache(BF, 200, 2, 16, 64)
    fill_cache(c, 1)
    dec = O.DecodeAttention(c, batch=2, heads=8, lib=seen)
    q = rand(2, 1, 8, 64, seed=2).to(DEV)
    bt, lens = torch.arange(200, dtype=torch.int32, device=DEV).view(2, 100), torch.tensor([1500, 900], dtype=torch.int32, device=DEV)
    want = dec(q, bt, lens)
    torch.cuda.synchronize()
    stream, graphs = torch.cuda.Stream(), []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            graphs.append((graph, dec(q, bt, lens)))
    with torch.cuda.stream(stream):
        late = dec(q, bt, lens)  # on the stream that was captured
    torch.cuda.synchronize()
    assert len(seen.workspaces) == len(set(seen.workspaces)) == 4
    for graph, out in graphs:
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(late, want)


@gpu
def test_graphs_of_one_handle_replayed_beside_each_other():
    c = make_cache(F8, 400, 2, 16, 128)
    fill_cache(c, 3)
    dec = O.DecodeAttention(c, batch=2, heads=16)
    bt = torch.arange(400, dtype=torch.int32, device=DEV).view(2, 200)
    calls = [(rand(2, 1, 16, 128, seed=4 + i).to(DEV), torch.tensor(n, dtype=torch.int32, device=DEV))
             for i, n in enumerate(([3100, 40], [900, 2000], [17, 3000]))]
    want = [dec(q, bt, n) for q, n in calls]
    torch.cuda.synchronize()
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    for q, n in calls[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(dec(q, bt, n))
    for _ in range(20):
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        eager = dec(calls[2][0], bt, calls[2][1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs + [eager], want))
    c.check()


# ------------------------------------------------------------ reports
@gpu
def test_check_waits_for_every_stream():
    c = make_cache(BF, 2, 2, 16, 64)
    dec = O.DecodeAttention(c, batch=1, heads=2)
    q = rand(1, 1, 2, 64).to(DEV)
    bt, n = torch.full((1, 2), 9, dtype=torch.int32, device=DEV), torch.full((1,), 5, dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        dec(q, bt, n)
    with pytest.raises(ValueError, match="block table"):
        c.check()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)  # tens of milliseconds
        dec(q, bt, n)
    with pytest.raises(ValueError, match="block table"):
        c.check()
    c.check()


@gpu
def test_reports_that_come_while_others_are_taken_stay():
    class Late(torch.Tensor):
        def item(self):
            bits = super().item()
            self.bitwise_or_(O.BAD_SLOT)  # as by a call that another thread enqueued
            return bits
    status = torch.full((1,), O.BAD_PAGE | O.BAD_LENGTH, dtype=torch.int32, device=DEV).as_subclass(Late)
    with pytest.raises(ValueError, match="block table.*lengths"):
        O.raise_faults(status)
    assert torch.Tensor.item(status) == O.BAD_SLOT
    O.raise_faults(torch.zeros((), dtype=torch.int32, device=DEV))


# ------------------------------------------------------------ autograd
@gpu
def test_rows_that_require_gradients_are_refused():
    x = rand(4, 2, 64).to(DEV)
    g = x.clone().requires_grad_()
    cu = torch.tensor([0, 4], dtype=torch.int32, device=DEV)
    c = make_cache(BF, 2, 2, 16, 64)
    pos, table = torch.arange(4, device=DEV), O.rotary_table(5, 64, device=DEV)
    dec = O.DecodeAttention(c, batch=1, heads=2)
    bt, n = torch.zeros(1, 2, dtype=torch.int32, device=DEV), torch.full((1,), 4, dtype=torch.int32, device=DEV)
    calls = [lambda a, t=t: O.attn_prompt(*(a if i == t else x for i in range(3)), cu, max_q=4) for t in range(3)]
    calls += [lambda a, t=t: O.rope_write(*(a if i == t else x for i in range(3)), pos, table, c, pos, keep_keys=True)
              for t in range(3)]
    calls += [lambda a: dec(a[None, :1], bt, n), lambda a: O.attn_prompt(x, x, x, cu, max_q=4, out=a),
              lambda a: O.rope_write(x, None, None, pos, table, q_out=a), lambda a: dec(x[None, :1], bt, n, out=a[None, :1]),
              lambda a: O.cache_read(c, bt, cu, total=4, v_out=a)]
    for call in calls:
        with pytest.raises(ValueError, match="backward"):
            call(g)
        with torch.no_grad():
            got = call(g)
        want = call(x.clone())
        for a, b in zip(got if isinstance(got, tuple) else [got], want if isinstance(want, tuple) else [want]):
            assert a is None and b is None or torch.equal(a, b)
    with pytest.raises(ValueError, match="gradients"):
        O.PagedCache(c.k.clone().requires_grad_(), c.v)


@gpu
def test_written_tensors_count_as_changed():
    """A backward pass that needs what a call has overwritten raises, as after torch's own in-place operations."""
    x = rand(4, 2, 64).to(DEV)
    cu = torch.tensor([0, 4], dtype=torch.int32, device=DEV)
    pos, table = torch.arange(4, device=DEV), O.rotary_table(5, 64, device=DEV)
    bt, n = torch.zeros(1, 2, dtype=torch.int32, device=DEV), torch.full((1,), 4, dtype=torch.int32, device=DEV)
    for kind in (BF, F8):
        c = make_cache(kind, 2, 2, 16, 64)
        dec, written = O.DecodeAttention(c, batch=1, heads=2, dtype=BF), [t for t in (c.k, c.v, c.k_scale, c.v_scale) if t is not None]
        out = x.clone()
        for call, changed in ((lambda: O.rope_write(x, x, x, pos, table, c, pos), written),
                              (lambda: O.rope_write(x, x, None, pos, table, q_out=out), [out]),
                              (lambda: O.rope_write(x, x, None, pos, table, k_out=out), [out]),
                              (lambda: O.cache_read(c, bt, cu, total=4, dtype=BF, k_out=out), [out]),
                              (lambda: O.cache_read(c, bt, cu, total=4, dtype=BF, v_out=out), [out]),
                              (lambda: O.attn_prompt(x, x, x, cu, max_q=4, out=out), [out]),
                              (lambda: dec(x[None, :1], bt, n, out=out[None, :1]), [out])):
            before = {id(t): t._version for t in (*written, out, x)}
            call()
            for t in (*written, out, x):
                assert (t._version > before[id(t)]) == any(t is s for s in changed)
    w = torch.ones(2, 2, 16, 64, dtype=BF, device=DEV, requires_grad=True)
    c = make_cache(BF, 2, 2, 16, 64)
    loss = (w * c.k).sum()
    O.rope_write(x, x, x, pos, table, c, pos)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


# ------------------------------------------------------------ grids
def test_longest_sequence_beyond_the_rows(fake):
    """max_q may be any bound: grids are those of at most all rows, also where the bound is the type's largest."""
    res = child(fake, """
        import struct
        PROMPT = struct.Struct("@3P6q4Pi2q7ifPN2P")

        def prompt(n_q, n_k, max_q, heads, kv_heads, dim, n_seqs=1, workspace=0):
            device()
            a = 1 << 44
            args = PROMPT.pack(a, a, a, heads * dim, dim, kv_heads * dim, dim, kv_heads * dim, dim, a, 0, a, a, n_seqs, n_q, n_k,
                               max_q, heads, kv_heads, dim, 0, 1, 0, 1.0, workspace, 1 << 40, 0, 0)
            lib.herschel_attn_prompt.argtypes = [ctypes.c_void_p]
            return lib.herschel_attn_prompt(args), log()
        for sizes in ((50, 50, 8, 2, 64), (4096, 4096, 32, 8, 128), (3000, 3000, 16, 16, 64), (700, 9000, 8, 2, 128),
                      (2000, 9000, 16, 2, 128)):
            n_q, n_k, heads, kv_heads, dim = sizes
            for most in (n_q, n_q + 1, 2**31 - 1, 2**31 - 100):
                for w in (0, 1 << 44):
                    out.append((n_q, most, prompt(n_q, n_k, most, heads, kv_heads, dim, workspace=w)))
    """)
    for i in range(0, len(res), 8):
        for w in (0, 1):
            want = res[i + w][2]
            assert want[0] == H.OK and launches(want[1])
            for n_q, most, got in res[i + w:i + 8:2]:
                assert got == want, (n_q, most, got, want)


# ------------------------------------------------------------ small values
@gpu
@pytest.mark.parametrize("power", [-60, -80, -88])
def test_small_values_scale(power):
    """Values times a power of two give outputs times it, down to near bf16's smallest: exponentials that leave room for
    sums of the largest values leave it below too.  The values are from 2^-10 on: with 2^-88, and 2^-30 for the largest
    weight, what a weight of 2^-8 of it adds is above 2^-140, a number with 9 places, and lesser ones make up less than
    2^-8 of an output."""
    by = 2.0 ** power
    q, k, v = rand(40, 4, 64, seed=1).to(DEV), rand(700, 2, 64, seed=2).to(DEV), (rand(700, 2, 64, seed=3).abs() + 0.5).to(DEV)
    for more in (0, 8000):
        qq = torch.cat([q, q.new_zeros(more, 4, 64)])
        starts = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, 40, 40 + more], [0, 700, 700]))
        starts = tuple(starts)
        a, b = (O.attn_prompt(qq, k, x, *starts, max_q=max(40, more))[:40].double() for x in (v, v * by))
        assert ((b / by - a).abs() <= 2.0 ** -7 * a).all()
    for kind in (BF, F8, I8):
        c = make_cache(kind, 64, 2, 16, 64)
        fill_cache(c, 1)
        dec = O.DecodeAttention(c, batch=1, heads=4, dtype=BF)
        bt, n = torch.arange(64, dtype=torch.int32, device=DEV)[None], torch.tensor([1000], dtype=torch.int32, device=DEV)
        if kind == BF:
            c.v.copy_(c.v.abs() + 0.5)
        else:  # magnitudes
            c.v.view(torch.uint8).bitwise_and_(0x7f)
        a = dec(q[:1][None], bt, n).double()
        (c.v if kind == BF else c.v_scale).mul_(by)
        b = dec(q[:1][None], bt, n).double()
        assert ((b / by - a).abs() <= 2.0 ** -7 * a).all(), kind


# ------------------------------------------------------------ weights over 8-bit caches
@gpu
@pytest.mark.parametrize("kind", [F8, I8], ids=str)
@pytest.mark.parametrize("lens,hq,hk,D,new", [([700, 3], 16, 1, 128, 1), ([4000], 8, 2, 64, 1), ([90, 200], 8, 2, 128, 4)], ids=str)
def test_decode_weights_over_codes_keep_two_parts(lens, hq, hk, D, new, kind):
    """Up to 16 rows of a key head, bf16 rows as well: a weight is rounded to 16 bits' worth of two parts, 2^-16, and
    the output once."""
    page = 16
    c = make_cache(kind, sum(-(-n // page) for n in lens) + 1, hk, page, D)
    fill_cache(c, 7)
    bt = paged(c, lens, 8)
    q = rand(len(lens), new, hq, D, seed=9)
    dec = O.DecodeAttention(c, batch=len(lens), heads=hq, new_tokens=new, dtype=BF)
    out, lse = dec(q.to(DEV), bt.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), return_lse=True)
    c.check()
    for b, (k, v) in enumerate(dense(c, bt, lens)):
        check_attention(out[b], lse[b], exact_attention(q[b], k, v, D ** -0.5, True, 0), BF, 2.0 ** -16, lens[b], D)


@gpu
@pytest.mark.parametrize("lens,hq,hk,D,new", [([700, 3], 16, 1, 128, 1), ([4000], 8, 2, 64, 1), ([90, 200], 8, 2, 128, 4)], ids=str)
def test_decode_weights_over_bf16_caches_keep_two_parts(lens, hq, hk, D, new):
    test_decode_weights_over_codes_keep_two_parts(lens, hq, hk, D, new, BF)


@gpu
def test_no_keys_at_all():
    """Rows without any key, over empty tensors and a block table without entries: 0, with a log sum of minus infinity."""
    none = torch.empty(0, 2, 64, dtype=BF, device=DEV)
    for n, heads in ((5, 4), (6000, 4), (1100, 64)):
        q = rand(n, heads, 64 if heads == 4 else 128).to(DEV)
        kv = none if heads == 4 else torch.empty(0, 2, 128, dtype=BF, device=DEV)
        cu_q, cu_k = (torch.tensor([0, x], dtype=torch.int32, device=DEV) for x in (n, 0))
        for causal in (True, False):
            out, lse = O.attn_prompt(q, kv, kv, cu_q, cu_k, max_q=n, causal=causal, return_lse=True)
            assert (out == 0).all() and (lse == -math.inf).all()
    c = make_cache(BF, 2, 2, 16, 64)
    dec = O.DecodeAttention(c, batch=3, heads=4)
    q = rand(3, 1, 4, 64).to(DEV)
    out, lse = dec(q, torch.empty(3, 0, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV), return_lse=True)
    c.check()
    assert (out == 0).all() and (lse == -math.inf).all()
