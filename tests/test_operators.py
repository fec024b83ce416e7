"""The reference operators (rotary write, cache read, prompt and decode
attention) against plain 64-bit implementations, and their refusals.

Tolerances are bounds, derived here and not fitted.  u is the unit roundoff of
the output's type (2^-8 for bfloat16 with its 8 significant bits, 2^-11 for
half with its 11: to nearest, half a last place), e that of the exponentials as
the second product takes them (the same, but 2^-16 where they go in two bf16
parts).  A row's output is sum p v / sum p:

* an error d of the scores changes each p by at most 2 d of itself (d < 0.1);
  f32 sums of D products of 16-bit numbers are off by (D + 8) 2^-24 sum |q k|;
* rounding p to e changes the output by at most e A, A = sum p |v| / sum p;
* f32 sums over n keys are off by n 2^-24 A; the result is rounded once, by u |o|.

So |o - exact| <= u |o| + (e + 2 d + (n + 16) 2^-23) A, and the rounding's u
times what the other terms added to |o|, which is under 2^-7 of them.
"""
from __future__ import annotations

import ctypes
import math
import os

import pytest
import torch

from paper_2609_40247_amd import herschel as H
from paper_2609_40247_amd import operators as O

BF, HF, F8, I8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8
U = {BF: 2.0 ** -8, HF: 2.0 ** -11}
gpu = pytest.mark.gpu
DEV = "cuda"


def named(value):
    """A parameter's name, the same in every process: some values print as addresses."""
    return "-".join(value) if isinstance(value, dict) else str(value)


def rand(*shape, seed=0, dtype=BF, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * gain).to(dtype)


# ------------------------------------------------------------ 64-bit definitions
def exact_rope(x, cs, layout, R):
    """x [T, h, D], cs [T, R/2, 2], in 64 bits; also the sum of the magnitudes that each element comes from."""
    x = x.double()
    y, mag = x.clone(), x.abs()
    c, s = cs[:, None, :, 0].double(), cs[:, None, :, 1].double()
    i = torch.arange(R // 2)
    ia, ib = (i, i + R // 2) if layout == "half" else (2 * i, 2 * i + 1)
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    mag[..., ia], mag[..., ib] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    return y, mag


def exact_attention(q, k, v, scale, causal, window):
    """q [n, h, D], k, v [m, g, D] -> out, lse, A = sum p |v| / sum p, largest sum |q k| scale of each row; 64 bits.
    Keys that a row does not see are left out, not multiplied by 0."""
    n, h, D = q.shape
    m, g = k.shape[:2]
    out, lse = torch.zeros(n, h, D, dtype=torch.float64), torch.full((n, h), -math.inf, dtype=torch.float64)
    A, S = torch.zeros_like(out), torch.zeros(n, h, dtype=torch.float64)
    for i in range(n):
        lo = max(0, i + m - n - window + 1) if window else 0
        hi = min(m, i + m - n + 1) if causal else m
        if hi <= lo:
            continue
        for x in range(h):
            kk, vv, qq = k[lo:hi, x * g // h].double(), v[lo:hi, x * g // h].double(), q[i, x].double()
            s = kk @ qq * scale
            z = torch.logsumexp(s, 0)
            p = torch.exp(s - z)
            out[i, x], lse[i, x], A[i, x] = p @ vv, z, p @ vv.abs()
            S[i, x] = (kk.abs() @ qq.abs()).max() * abs(scale)
    return out, lse, A, S


def check_attention(out, lse, ref, dtype, e, n_keys, D):
    o, l, A, S = ref
    d = (D + 8) * 2.0 ** -24 * S
    tol = U[dtype] * o.abs() + (1 + 2.0 ** -7) * (e + 2 * d[..., None] + (n_keys + 16) * 2.0 ** -23) * A + 1e-30
    if dtype == HF:
        tol = tol + 2.0 ** -25  # half's smallest step
    got = out.double().cpu()
    bad = torch.isnan(o) | torch.isinf(o)
    assert torch.equal(torch.isnan(got), torch.isnan(o))
    assert torch.equal(got[bad & ~torch.isnan(o)], o[bad & ~torch.isnan(o)])
    over = ((got - o).abs() - tol)[~bad]
    assert over.numel() == 0 or over.max() <= 0, (over.max(), (got - o)[~bad].abs().max())
    if lse is not None:
        got = lse.double().cpu()
        dead = l == -math.inf
        assert torch.equal(got == -math.inf, dead)
        live = ~dead & ~torch.isnan(l)
        assert ((got - l).abs()[live] <= (d + (n_keys + 16) * 2.0 ** -23 + 2.0 ** -22 * l.abs())[live]).all()


# ------------------------------------------------------------ rotary write
def scatter_slots(T, n_pages, page, seed):
    return torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(seed))[:T]


def make_cache(kind, n_pages, heads, page, D, fill=None):
    c = O.PagedCache.allocate(n_pages, heads, page, D, kind, DEV)
    if fill is not None:
        for t in (c.k, c.v):
            t.view(torch.uint8).fill_(fill)
        if c.quantised:
            c.k_scale.fill_(math.nan)
            c.v_scale.fill_(math.nan)
    return c


def rows_of(c, part):
    """The cache's rows in slot order, [slots, heads, D] codes and [slots, heads] scales, on the host."""
    t = getattr(c, part)
    t = (t.view(torch.uint8).cpu().view(t.dtype) if t.element_size() == 1 else t.cpu())
    f = t.float() if t.dtype != F8 else t.to(torch.float32)
    f = f.transpose(1, 2).reshape(-1, c.n_heads, c.head_dim)
    s = getattr(c, part + "_scale")
    return f, None if s is None else s.cpu().transpose(1, 2).reshape(-1, c.n_heads)


def check_stored(c, part, slots, y, mag, dtype):
    """Rows y (64 bits, each off by at most 2^-22 mag in 32 bits) as the cache holds them."""
    f, s = rows_of(c, part)
    f = f[slots].double()
    if not c.quantised:
        assert ((f - y).abs() <= U[dtype] * y.abs() + 2.0 ** -22 * mag + (2.0 ** -25 if dtype == HF else 0)).all()
        return
    M = 448.0 if c.k.dtype == F8 else 127.0
    s = s[slots].double()
    want = (y.abs().amax(-1) / M).clamp_min(2.0 ** -100)
    assert ((s - want).abs() <= 2.0 ** -22 * (want + mag.amax(-1) / M)).all()
    s = s[..., None]
    half = s / 2 if c.k.dtype == I8 else torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * s)  # half a step of the code
    assert ((f * s - y).abs() <= half * (1 + 2.0 ** -20) + 2.0 ** -20 * (mag + s * M * 2.0 ** -2)).all()
    assert (f.abs() <= M).all()


ROPE_CASES = [  # tokens, q heads, kv heads, D, R, layout, type, cache, page, strided
    (1, 8, 2, 128, 128, "half", BF, BF, 16, False),
    (37, 8, 2, 128, 128, "half", BF, F8, 64, True),
    (33, 5, 1, 128, 64, "half", HF, I8, 32, True),
    (65, 4, 4, 64, 32, "interleaved", HF, HF, 16, False),
    (300, 20, 4, 64, 64, "interleaved", BF, I8, 256, True),
    (130, 32, 8, 128, 128, "half", BF, F8, 64, True),
    (513, 32, 8, 128, 32, "interleaved", BF, F8, 128, False),
    (19, 3, 3, 256, 256, "half", BF, F8, 16, True),
    (7, 6, 2, 80, 80, "half", HF, I8, 16, False),
    (21, 6, 2, 96, 96, "half", BF, F8, 16, False),
    (9, 3, 1, 36, 20, "half", BF, F8, 16, False),
    (11, 4, 2, 250, 130, "interleaved", HF, I8, 32, False),
    (5, 2, 2, 64, 0, "half", BF, I8, 16, False),
    (40, 0, 2, 64, 64, "half", BF, F8, 16, False),
    (40, 6, 0, 64, 64, "half", BF, None, 16, False),
    (40, 6, 3, 128, 64, "half", HF, None, 16, True),
]


@gpu
@pytest.mark.parametrize("case", ROPE_CASES, ids=str)
def test_rope_write(case):
    T, hq, hk, D, R, layout, dtype, kind, page, strided = case
    heads = hq + 2 * max(hk, 1)
    x = rand(T, heads, D, seed=1, dtype=dtype, gain=3.0)
    x[0] *= 0.0  # a row of zeros
    if not strided:
        q, k, v = x[:, :hq].contiguous(), x[:, hq:hq + hk].contiguous(), x[:, hq + hk:hq + 2 * hk].contiguous()
        q, k, v = q.to(DEV), k.to(DEV), v.to(DEV)
    else:
        d = x.to(DEV)
        q, k, v = d[:, :hq], d[:, hq:hq + hk], d[:, hq + hk:hq + 2 * hk]
    q, k, v = q if hq else None, k if hk else None, v if hk and kind else None
    pos = torch.randint(0, 5000, (T,), generator=torch.Generator().manual_seed(3))
    table = O.rotary_table(5000, R, device=DEV)
    n_pages = T // page + 3
    cache = make_cache(kind, n_pages, hk, page, D, fill=0x11) if kind else None
    slots = scatter_slots(T, n_pages, page, 4)
    if T > 20:
        slots[7] = -1
    qo, ko = O.rope_write(q, k, v, pos.to(DEV), table, cache, slots.to(DEV) if kind else None, layout=layout,
                          keep_keys=True)
    torch.cuda.synchronize()
    cs = table.cpu()[pos]
    for name, inp, got in (("q", x[:, :hq], qo), ("k", x[:, hq:hq + hk], ko)):
        if got is None:
            continue
        y, mag = exact_rope(inp, cs, layout, R)
        err = (got.double().cpu() - y).abs()
        assert (err <= U[dtype] * y.abs() + 2.0 ** -22 * mag + (2.0 ** -25 if dtype == HF else 0)).all(), name
    if cache is None:
        return
    cache.check()
    kept = slots >= 0
    y, mag = exact_rope(x[:, hq:hq + hk], cs, layout, R)
    check_stored(cache, "k", slots[kept], y[kept], mag[kept], dtype)
    yv = x[:, hq + hk:hq + 2 * hk].double()
    check_stored(cache, "v", slots[kept], yv[kept], torch.zeros_like(yv[kept]), dtype)
    # rows that no token names are as they were
    rest = torch.ones(n_pages * page, dtype=torch.bool)
    rest[slots[kept]] = False
    for part in ("k", "v"):
        t = getattr(cache, part).view(torch.uint8).cpu().transpose(1, 2).reshape(n_pages * page, -1)
        assert (t[rest] == 0x11).all()


@gpu
def test_rope_in_place_and_views():
    """q rotated onto itself, and rows at addresses that no 16-byte load fits."""
    T, h, D = 50, 6, 64
    table = O.rotary_table(200, D, device=DEV)
    pos = torch.arange(T, device=DEV) * 3
    x = rand(T, h, D, seed=5)
    want, mag = exact_rope(x, table.cpu()[pos.cpu()], "half", D)
    bound = U[BF] * want.abs() + 2.0 ** -22 * mag
    a = x.to(DEV)
    out, _ = O.rope_write(a, None, None, pos, table, q_out=a)
    assert out is a and ((a.double().cpu() - want).abs() <= bound).all()
    flat = torch.zeros(T * h * (D + 3) + 1, dtype=BF, device=DEV)
    odd = flat[1:].view(T, h, D + 3)[:, :, :D]
    odd.copy_(x.to(DEV))
    out, _ = O.rope_write(odd, None, None, pos, table, q_out=odd)
    assert ((odd.double().cpu() - want).abs() <= bound).all()


@gpu
@pytest.mark.parametrize("kind", [F8, I8])
@pytest.mark.parametrize("D,R", [(128, 128), (36, 20)])
def test_rows_that_are_not_finite(kind, D, R):
    """A row with an infinity or a NaN reads back as NaN, its neighbours are untouched; largest and smallest rows hold."""
    T = 6
    x = rand(T, 3, D, seed=6)
    x[1, 1, D - 1] = math.inf
    x[2, 2, 3] = math.nan
    x[3] = torch.where(x[3] > 0, 3.38e38, -3.38e38).to(BF)
    x[4] *= 1e-37
    d = x.to(DEV)
    cache = make_cache(kind, 1, 1, 16, D)
    O.rope_write(d[:, :1], d[:, 1:2], d[:, 2:], torch.zeros(T, dtype=torch.int64, device=DEV),
                 O.rotary_table(1, R, device=DEV), cache, torch.arange(T, device=DEV))
    fk, sk = rows_of(cache, "k")
    fv, sv = rows_of(cache, "v")
    for t in range(T):
        for f, s, bad, row in ((fk, sk, t == 1, x[t, 1]), (fv, sv, t == 2, x[t, 2])):
            if bad:
                assert math.isnan(s[t, 0]) and (f[t, 0] == 0).all()
            else:
                M = 448.0 if kind == F8 else 127.0
                step = max(row.double().abs().max().item() / M, 2.0 ** -100)
                err = (f[t, 0].double() * s[t, 0].double() - row.double()).abs()
                assert (err <= 2.0 ** -4 * row.double().abs() * 1.001 + step * 0.501).all()


@gpu
@pytest.mark.parametrize("D", [64, 36])
def test_rope_faults_are_reported(D):
    T = 4
    d = rand(T, 3, D, seed=7).to(DEV)
    table = O.rotary_table(10, D // 4 * 2, device=DEV)
    cache = make_cache(I8, 2, 1, 16, D, fill=0x11)

    def go(pos, slots):
        return O.rope_write(d[:, :1], d[:, 1:2], d[:, 2:], torch.tensor(pos, device=DEV), table, cache,
                            torch.tensor(slots, device=DEV), keep_keys=True)
    go([0, 1, 2, 9], [0, 1, 2, 31])
    cache.check()
    go([0, 1, 2, 3], [0, 1, 32, -5])
    with pytest.raises(ValueError, match="slot"):
        cache.check()
    cache.check()  # cleared
    before = cache.k.clone()
    for bad in (10, -1, 1 << 40):
        q, k = go([bad, 1, 2, 3], [5, -1, -1, -1])
        with pytest.raises(ValueError, match="position"):
            cache.check()
        R = D // 4 * 2
        assert torch.isnan(q[0, :, :R]).all() and torch.isnan(k[0, :, :R]).all()
        assert torch.isfinite(q[1:]).all()
    assert torch.equal(cache.k, before)


def test_rotary_table():
    t = O.rotary_table(100, 8, base=100.0, stretch=4.0, device="cpu")
    assert t.shape == (100, 4, 2) and t.dtype == torch.float32
    for i in range(4):
        for p in (0, 1, 99):
            a = p / 4 * 100.0 ** (-2 * i / 8)
            assert abs(t[p, i, 0].item() - math.cos(a)) < 1e-7 and abs(t[p, i, 1].item() - math.sin(a)) < 1e-7
    # blended: the fastest pair as trained, the slowest compressed
    b = O.rotary_table(5000, 64, stretch=8.0, blend=(4096, 1, 32), device="cpu")
    one, eight = O.rotary_table(5000, 64, device="cpu"), O.rotary_table(5000, 64, stretch=8.0, device="cpu")
    assert torch.equal(b[:, 0], one[:, 0]) and torch.equal(b[:, -1], eight[:, -1])
    # angles in 64 bits: far positions stay exact
    far = O.rotary_table(131_072, 2, device="cpu")[131_071, 0]
    assert abs(far[0].item() - math.cos(131_071)) < 1e-7
    for bad in (dict(rotary_dim=3), dict(rotary_dim=4, stretch=0), dict(rotary_dim=4, blend=(4096, 2, 1)),
                dict(rotary_dim=4, base=-1)):
        with pytest.raises(ValueError):
            O.rotary_table(10, device="cpu", **bad)


# ------------------------------------------------------------ cache read
def fill_cache(c, seed, stale=None):
    """Random contents; on the device, so that large caches are quick."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    for t, s in ((c.k, c.k_scale), (c.v, c.v_scale)):
        if c.quantised:
            codes = torch.randint(0, 255, t.shape, generator=g, device=DEV, dtype=torch.int32)
            if t.dtype == F8:
                codes = torch.where((codes & 127) == 127, codes - 1, codes)  # no NaN
            t.view(torch.uint8).copy_(codes.to(torch.uint8))
            s.copy_(torch.rand(s.shape, generator=g, device=DEV) * (2.0 / (448 if t.dtype == F8 else 127)) + 1e-4)
        else:
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))


def paged(c, lens, seed, spare=2):
    """A block table for sequences of these lengths; entries beyond a sequence's pages are garbage."""
    pages = [-(-n // c.page_size) for n in lens]
    order = torch.randperm(c.n_pages, generator=torch.Generator().manual_seed(seed)).int()
    assert sum(pages) <= c.n_pages
    bt = torch.full((len(lens), max(pages) + spare), -7, dtype=torch.int32)
    bt[:, 1::2] = 2 ** 31 - 1
    at = 0
    for b, n in enumerate(pages):
        bt[b, :n] = order[at:at + n]
        at += n
    return bt


def dense(c, bt, lens):
    """Keys and values of each sequence from the cache, in 64 bits on the host."""
    res = []
    for b, n in enumerate(lens):
        ids = bt[b, :-(-n // c.page_size)].long().to(DEV)
        pair = []
        for t, s in ((c.k, c.k_scale), (c.v, c.v_scale)):
            x = (t.view(torch.uint8)[ids].cpu().view(t.dtype).float() if t.element_size() == 1 else t[ids].cpu()).double()
            if s is not None:
                x = x * s[ids].cpu().double()[..., None]
            pair.append(x.transpose(1, 2).reshape(-1, c.n_heads, c.head_dim)[:n])
        res.append(pair)
    return res


@gpu
@pytest.mark.parametrize("kind,dtype", [(BF, BF), (HF, HF), (F8, BF), (F8, HF), (I8, BF), (I8, HF)], ids=str)
@pytest.mark.parametrize("heads,page,D,lens", [(1, 16, 64, [1]), (3, 32, 128, [0, 33, 1, 0, 64, 17]),
                                               (8, 256, 128, [700, 5]), (2, 64, 48, [65, 130]), (1, 16, 256, [50])],
                         ids=str)
def test_cache_read(kind, dtype, heads, page, D, lens):
    c = make_cache(kind, sum(-(-n // page) for n in lens) + 3, heads, page, D)
    fill_cache(c, 1)
    bt = paged(c, lens, 2)
    cu = torch.tensor([0] + lens).cumsum(0).int().to(DEV)
    k, v = O.cache_read(c, bt.to(DEV), cu, total=sum(lens), dtype=dtype)
    c.check()
    for got, part in ((k, 0), (v, 1)):
        want = torch.cat([x[part] for x in dense(c, bt, lens)])
        tol = U[dtype] * want.abs() + (2.0 ** -25 if dtype == HF else 0) if c.quantised else 0 * want
        assert ((got.double().cpu() - want).abs() <= tol).all()


@gpu
def test_cache_read_faults():
    c = make_cache(BF, 4, 2, 16, 64)
    fill_cache(c, 3)
    cu = torch.tensor([0, 20, 40], dtype=torch.int32, device=DEV)
    for bad in (4, -1, 2 ** 31 - 1):
        bt = torch.tensor([[0, 1], [2, bad]], dtype=torch.int32, device=DEV)
        k, _ = O.cache_read(c, bt, cu, total=40)
        with pytest.raises(ValueError, match="block table"):
            c.check()
        assert (k[36:] == 0).all() and torch.equal(k[20:36], c.k[2].transpose(0, 1))
    bt = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device=DEV)
    k, _ = O.cache_read(c, bt, cu, total=43)  # rows that no sequence has
    with pytest.raises(ValueError, match="lengths"):
        c.check()
    assert (k[40:] == 0).all()
    k, _ = O.cache_read(c, bt[:, :1].contiguous(), cu, total=40)  # longer than the table has room for
    with pytest.raises(ValueError, match="lengths"):
        c.check()
    assert (k[16:20] == 0).all()


@gpu
def test_offsets_beyond_32_bits():
    """A cache of over 2^32 bytes and elements: its last pages written, read and attended to."""
    heads, page, D = 8, 256, 128
    n_pages = (1 << 32) // (heads * page * D) + 5  # elements of k pass 2^32
    k = torch.empty(n_pages, heads, page, D, dtype=I8, device=DEV)
    v = torch.empty_like(k)
    ks, vs = (torch.empty(n_pages, heads, page, device=DEV) for _ in range(2))
    c = O.PagedCache(k, v, ks, vs)
    T = 300
    ids = torch.tensor([n_pages - 1, n_pages - 3], dtype=torch.int32)
    x = rand(T, 3 * heads, D, seed=8)
    d = x.to(DEV)
    tok = torch.arange(T)
    slots = ids[tok // page].long() * page + tok % page
    table = O.rotary_table(T, D, device=DEV)
    qo, _ = O.rope_write(d[:, :heads], d[:, heads:2 * heads], d[:, 2 * heads:], tok.to(DEV), table, c, slots.to(DEV))
    bt = ids[None].to(DEV)
    kr, vr = O.cache_read(c, bt, torch.tensor([0, T], dtype=torch.int32, device=DEV), total=T)
    c.check()
    y, _ = exact_rope(x[:, heads:2 * heads], table.cpu(), "half", D)
    for got, want in ((kr, y), (vr, x[:, 2 * heads:].double())):
        step = want.abs().amax(-1, keepdim=True) / 127
        assert ((got.double().cpu() - want).abs() <= 0.501 * step + U[BF] * want.abs() + 1e-6).all()
    ref_k, ref_v = dense(c, ids[None], [T])[0]
    dec = O.DecodeAttention(c, batch=1, heads=heads, dtype=BF)
    o = dec(qo[-1:][None], bt, torch.tensor([T], dtype=torch.int32, device=DEV))
    ref = exact_attention(qo[-1:].cpu(), ref_k, ref_v, D ** -0.5, True, 0)
    check_attention(o[0], None, ref, BF, U[BF], T, D)


# ------------------------------------------------------------ prompts
def run_prompt(nq, nk, hq, hk, D, dtype, causal, window, strided=False, seed=0, edit=None, gain=1.0, scale=None):
    Tq, Tk = sum(nq), sum(nk)
    q = rand(Tq, hq, D, seed=seed + 1, dtype=dtype, gain=gain)
    k = rand(Tk, hk, D, seed=seed + 2, dtype=dtype, gain=gain)
    v = rand(Tk, hk, D, seed=seed + 3, dtype=dtype)
    if edit:
        edit(q, k, v)
    dq, dk, dv = q.to(DEV), k.to(DEV), v.to(DEV)
    if strided == "rows":  # slices of wider rows, heads not adjacent
        dq, dk, dv = (torch.zeros(t.shape[0], 2 * t.shape[1] + 1, D + 8, dtype=dtype, device=DEV)[:, 1::2, 8:]
                      .copy_(t) for t in (dq, dk, dv))
    if strided == "odd":  # addresses that no 16-byte load fits
        dq, dk, dv = (torch.zeros(t.numel() // D * (D + 1) + 1, dtype=dtype, device=DEV)[1:]
                      .view(t.shape[0], t.shape[1], D + 1)[:, :, :D].copy_(t) for t in (dq, dk, dv))
    cu = [torch.tensor([0] + list(n)).cumsum(0).int().to(DEV) for n in (nq, nk)]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = O.attn_prompt(dq, dk, dv, *cu, max_q=max(nq), scale=scale, causal=causal, window=window,
                             return_lse=True, status=status)
    assert status.item() == 0
    at_q = at_k = 0
    for n, m in zip(nq, nk):
        ref = exact_attention(q[at_q:at_q + n], k[at_k:at_k + m], v[at_k:at_k + m], D ** -0.5 if scale is None else scale,
                              causal, window)
        check_attention(out[at_q:at_q + n], lse[at_q:at_q + n], ref, dtype, U[dtype], m, D)
        at_q, at_k = at_q + n, at_k + m


PROMPT_CASES = [  # queries, keys, heads, kv heads, D, causal, window
    ([1], [1], 1, 1, 64, True, 0),
    ([1, 2, 0, 31, 33], None, 4, 2, 128, True, 0),
    ([64, 65, 127, 128, 129], None, 2, 1, 64, True, 0),
    ([200], [200], 5, 1, 128, False, 0),
    ([3, 70], [200, 70], 8, 2, 128, True, 0),
    ([150], [257], 2, 2, 64, True, 40),
    ([130, 20], [130, 300], 4, 4, 128, True, 1),
    ([90], [100], 2, 1, 128, False, 17),
    ([100, 5, 140], [40, 0, 139], 2, 1, 64, True, 0),      # queries before the first key, no key at all
    ([100, 5], [40, 0], 2, 1, 128, False, 0),
    ([140], [30], 2, 2, 64, True, 20),
    ([1, 1, 1], [500, 3, 129], 16, 2, 128, True, 0),
]


@gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
@pytest.mark.parametrize("case", PROMPT_CASES, ids=str)
def test_attn_prompt(case, dtype):
    nq, nk, hq, hk, D, causal, window = case
    run_prompt(nq, nk or nq, hq, hk, D, dtype, causal, window)


RAGGED_CASES = [  # queries, keys, heads, kv heads, D, causal, window
    ([600] + [1, 0, 3, 17] * 2, None, 8, 2, 64, True, 0),
    ([0, 0, 5, 0, 90, 1], [7, 0, 5, 0, 200, 0], 10, 2, 128, True, 40),
    ([(7 * i) % 11 for i in range(150)], None, 2, 2, 64, True, 0),             # beyond 64 sequences
    ([0] * 130 + [70] + [0] * 3 + [33], None, 3, 1, 128, False, 0),
    ([0] * 70 + [70] + [1, 0, 9] * 16 + [33], None, 3, 1, 128, False, 0),      # the second 64
    ([200] + [2] * 63 + [150] + [0] * 20, None, 4, 1, 64, True, 60),
]


@gpu
@pytest.mark.parametrize("case", RAGGED_CASES, ids=lambda c: f"{len(c[0])}-{sum(c[0])}-{c[4]}")
def test_attn_prompt_ragged(case):
    """Packed sequences of very different lengths, empty ones between and at the ends."""
    nq, nk, hq, hk, D, causal, window = case
    run_prompt(nq, nk or nq, hq, hk, D, BF, causal, window)


@gpu
def test_attn_prompt_faults_of_ragged_sequences():
    """Starts that fall, exceed the rows or are negative among many sequences: reported, every row still written."""
    q = rand(300, 4, 64).to(DEV)
    good = [0, 1, 1, 4, 200] + [200 + 25 * i for i in range(1, 5)]

    def go(cu_q, cu_k, max_q=196):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        out = torch.full_like(q, math.nan)
        O.attn_prompt(q, q[:, :2], q[:, 2:], torch.tensor(cu_q, dtype=torch.int32, device=DEV),
                      torch.tensor(cu_k, dtype=torch.int32, device=DEV), max_q=max_q, status=status, out=out)
        return status.item(), out
    bits, want = go(good, good)
    assert bits == 0 and torch.isfinite(want).all()
    for i, value in ((2, 0), (4, 2), (4, -9), (8, 500), (3, 2 ** 31 - 1)):
        bad = list(good)
        bad[i] = value
        assert go(good, bad)[0] == O.BAD_LENGTH
        bits, out = go(bad, good, max_q=300)
        assert bits == O.BAD_LENGTH and torch.isfinite(out).all()
    bits, out = go(good, good, max_q=100)
    assert bits == O.BAD_LENGTH and torch.equal(out[:104], want[:104]) and torch.equal(out[200:], want[200:])


@gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
@pytest.mark.parametrize("case", PROMPT_CASES, ids=str)
def test_attn_prompt_among_many_rows(case, dtype):
    """The same beside a long sequence that sees no key: calls of few rows and of many are worked on differently."""
    nq, nk, hq, hk, D, causal, window = case
    run_prompt(nq + [30_000 // hq], (nk or nq) + [0], hq, hk, D, dtype, causal, window)


@gpu
@pytest.mark.parametrize("strided", ["rows", "odd"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("more", [0, 8000])
def test_attn_prompt_strides(strided, D, more):
    run_prompt([70, 33, more], [70, 90, 0], 4, 2, D, BF, True, 0, strided=strided)


@gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
def test_attn_prompt_hidden_values_have_no_effect(D, dtype):
    """Infinities and NaN in keys and values reach the rows that see them, as they would in 64 bits, and no other;
    large and rising scores, whose maximum is looked at again and again, keep their precision."""
    def edit(q, k, v):
        v[100, 0, 5] = math.nan
        v[101, 1, 6] = math.inf
        v[102, 0, 7] = -math.inf
        k[149, 1] = math.nan
    for more in (0, 8000):
        run_prompt([150, more], [150, 0], 4, 2, D, dtype, True, 0, edit=edit)
        run_prompt([40, more], [200, 0], 4, 2, D, dtype, True, 30, edit=edit)  # behind the window

    def rising(q, k, v):
        k *= torch.linspace(0, 6, k.shape[0])[:, None, None].to(k.dtype)
        q[:, :, 0] = 4
        k[:, :, 0] = torch.linspace(-30, 30, k.shape[0])[:, None].to(k.dtype)
    for more in (0, 16_000):
        run_prompt([180, more], [180, 0], 2, 1, D, dtype, True, 0, edit=rising, scale=0.25)
        run_prompt([40, more], [150, 0], 2, 1, D, dtype, False, 0, scale=0.0)
        run_prompt([40, more], [150, 0], 2, 1, D, dtype, True, 0, scale=-0.1)


LONG_CASES = [  # queries, keys, heads, kv heads, causal, window, values that are not finite
    ([1500, 1029], None, 64, 8, True, 0, False),
    ([1024, 1300], [2000, 1300], 64, 4, True, 700, False),
    ([1100, 1100], [1100, 900], 64, 64, True, 0, True),
    ([1030, 1026], [1030, 1700], 64, 16, False, 0, False),
    ([1030, 1026], [1200, 70], 65, 5, False, 90, True),
]


@gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
@pytest.mark.parametrize("case", LONG_CASES, ids=str)
def test_attn_prompt_long(case, dtype):
    """Enough rows and heads for the larger workgroups: chosen rows of chosen heads against 64 bits."""
    nq, nk, hq, hk, causal, window, odd = case
    nk, D = nk or nq, 128
    q, k, v = (rand(sum(n), h, D, seed=11 + i, dtype=dtype) for i, (n, h) in enumerate(((nq, hq), (nk, hk), (nk, hk))))
    if odd:
        v[700, 0, 3], v[701, 0, 4], k[705, hk - 1] = math.inf, math.nan, math.nan
    cu = [torch.tensor([0] + list(n)).cumsum(0).int().to(DEV) for n in (nq, nk)]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = O.attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), *cu, max_q=max(nq), causal=causal, window=window,
                             return_lse=True, status=status)
    assert status.item() == 0
    out, lse = out.cpu(), lse.cpu()
    heads = sorted({0, hq // hk - 1, hq // 2, hq - 1})
    at_q = at_k = 0
    for n, m in zip(nq, nk):
        for i in sorted({0, 1, 31, 32, 63, 255, 256, 511, 700, 701, 705, n - 65, n - 2, n - 1}):
            hi = max(0, min(m, i + m - n + 1)) if causal else m  # as the last row of a shorter sequence
            lo = max(0, i + m - n - window + 1) if window else 0
            for h in heads:
                g = h * hk // hq
                ref = exact_attention(q[at_q + i:at_q + i + 1, h:h + 1], k[at_k + lo:at_k + max(lo, hi), g:g + 1],
                                      v[at_k + lo:at_k + max(lo, hi), g:g + 1], D ** -0.5, False, 0)
                check_attention(out[at_q + i:at_q + i + 1, h:h + 1], lse[at_q + i:at_q + i + 1, h:h + 1], ref, dtype,
                                U[dtype], m, D)
        at_q, at_k = at_q + n, at_k + m


PART_CASES = [  # queries, keys, heads, kv heads, D, causal, window, strided
    ([3, 40, 0], [2100, 6000, 9], 8, 2, 128, True, 0, False),
    ([64], [2500], 4, 1, 64, True, 0, "rows"),
    ([1, 70], [4100, 30], 5, 1, 64, False, 1000, False),
    ([33], [9000], 16, 4, 128, True, 3, "odd"),             # parts without a key
]
MANY_PART_CASES = [  # workgroups of 128 rows
    ([530], [5200], 16, 2, 128, True, 0, False, BF),
    ([1900, 100], [8300, 100], 11, 11, 64, True, 2600, "rows", HF),
    ([1350], [4100], 8, 1, 128, False, 0, "odd", BF),
]


def splits_of(nq, nk, hq, hk, D):
    """Bytes of workspace in parts of a row."""
    size = ctypes.c_size_t(0)
    assert lib().herschel_attn_prompt_workspace(len(nq), sum(nq), sum(nk), max(nq), hq, hk, D, ctypes.byref(size)) == H.OK
    return size.value / (sum(nq) * hq * (D + 4) * 4)


def test_attn_prompt_workspace_is_for_few_rows_over_many_keys():
    for nq, nk, hq, hk, D, *_ in PART_CASES + MANY_PART_CASES:
        assert splits_of(nq, nk, hq, hk, D) in range(2, 17)
    assert splits_of([4096], [4096], 32, 8, 128) == 0
    assert splits_of([100], [100], 32, 8, 128) == 0
    size = ctypes.c_size_t(0)
    for bad in ((0, 1, 1, 1, 1, 1, 64), (1, -1, 1, 1, 1, 1, 64), (1, 1, 1, 1, 3, 2, 64), (1, 1, 1, 1, 1, 1, 96)):
        assert lib().herschel_attn_prompt_workspace(*bad, ctypes.byref(size)) == H.EINVAL
    assert lib().herschel_attn_prompt_workspace(1, 1, 1, 1, 1, 1, 64, None) == H.EINVAL
    assert lib().herschel_attn_prompt(ctypes.byref(prompt_args(workspace=FAKE + 8, workspace_bytes=1 << 30))) == H.EWORKSPACE


@gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
@pytest.mark.parametrize("case", PART_CASES, ids=str)
def test_attn_prompt_in_parts(case, dtype):
    nq, nk, hq, hk, D, causal, window, strided = case
    run_prompt(nq, nk, hq, hk, D, dtype, causal, window, strided=strided)


@gpu
@pytest.mark.parametrize("case", MANY_PART_CASES, ids=str)
def test_attn_prompt_of_many_rows_in_parts(case):
    nq, nk, hq, hk, D, causal, window, strided, dtype = case
    run_prompt(nq, nk, hq, hk, D, dtype, causal, window, strided=strided)


@gpu
def test_attn_prompt_in_parts_hidden_values_have_no_effect():
    def edit(q, k, v):
        v[2100, 0, 5] = math.nan
        v[4099, 0, 6] = math.inf
        v[10, 1, 7] = -math.inf
        k[4098, 1] = math.nan
    run_prompt([40], [4100], 4, 2, 128, BF, True, 0, edit=edit)
    run_prompt([40], [4100], 4, 2, 64, HF, True, 4000, edit=edit)
    run_prompt([1400], [4100], 8, 2, 128, HF, True, 0, edit=edit)


@gpu
def test_attn_prompt_in_parts_in_a_graph_and_without_workspace(monkeypatch):
    q, k, v = (rand(n, h, 128, seed=i).to(DEV) for i, (n, h) in enumerate(((50, 8), (5000, 2), (5000, 2))))
    cu_q, cu_k = (torch.tensor([0, n], dtype=torch.int32, device=DEV) for n in (50, 5000))
    call = lambda: O.attn_prompt(q, k, v, cu_q, cu_k, max_q=50)
    eager = call()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = call()
    for step in range(4):
        q.copy_(rand(50, 8, 128, seed=20 + step))
        eager = call()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
    monkeypatch.setattr(O, "_prompt_workspace", lambda *a: 0)
    whole = call()
    ref = exact_attention(q.cpu(), k.cpu(), v.cpu(), 128 ** -0.5, True, 0)
    for got in (eager, whole):
        check_attention(got, None, ref, BF, U[BF], 5000, 128)


@gpu
def test_attn_prompt_faults():
    q = rand(40, 2, 64).to(DEV)

    def go(cu_q, cu_k, max_q=40):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        out = torch.zeros_like(q)
        O.attn_prompt(q, q, q, torch.tensor(cu_q, dtype=torch.int32, device=DEV),
                      torch.tensor(cu_k, dtype=torch.int32, device=DEV), max_q=max_q, status=status, out=out)
        return status, out
    status, _ = go([0, 20, 40], [0, 20, 40])
    assert status.item() == 0
    for bad in (([0, 20, 41], [0, 20, 40]), ([0, 20, 40], [0, 20, 2 ** 31 - 1]), ([0, 20, 10], [0, 20, 40]),
                ([0, -5, 40], [0, 20, 40])):
        status, out = go(*bad)
        assert status.item() == O.BAD_LENGTH and torch.isfinite(out).all()
        with pytest.raises(ValueError, match="lengths"):
            O.raise_faults(status)
        assert status.item() == 0
    status, out = go([0, 40], [0, 40], max_q=7)
    assert status.item() == O.BAD_LENGTH and (out[7:] == 0).all() and (out[:7] != 0).any()
    assert O.attn_prompt(q[:0], q[:0], q[:0], torch.tensor([0, 0], dtype=torch.int32, device=DEV), max_q=0).shape == (0, 2, 64)


@gpu
@pytest.mark.parametrize("case", [([100, 5, 140], [40, 0, 139], 2, 1, 64, False), ([300], [200], 4, 4, 128, False),
                                  ([300], [200], 4, 1, 128, True)], ids=str)
def test_attn_prompt_widest_windows(case):
    """Windows that reach below the first key by nearly 2^31: the same as none, also with more queries than keys."""
    nq, nk, hq, hk, D, causal = case
    for window in (2 ** 31 - 1, 2 ** 31 - 100):
        run_prompt(nq, nk, hq, hk, D, BF, causal, window)


# ------------------------------------------------------------ decode
def run_decode(lens, hq, hk, D, dtype, kind, page, new=1, window=0, edit=None, strided=False, seed=0, scale=None):
    B = len(lens)
    c = make_cache(kind, sum(-(-n // page) for n in lens) + 3, hk, page, D)
    fill_cache(c, seed)
    bt = paged(c, lens, seed + 1)
    if edit:
        edit(c, bt)
    q = rand(B, new, hq, D, seed=seed + 2, dtype=dtype)
    dq = q.to(DEV)
    if strided:
        dq = torch.zeros(B, new + 1, hq + 2, D + 1, dtype=dtype, device=DEV)[:, :new, 1:hq + 1, 1:].copy_(dq)
    dec = O.DecodeAttention(c, batch=B + 3, heads=hq, new_tokens=new, dtype=dtype)
    sl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    out, lse = dec(dq, bt.to(DEV), sl, scale=scale, window=window, return_lse=True)
    c.check()
    rounded = U[dtype] if not c.quantised else U[BF] if dtype == BF else 2.0 ** -16
    for b, (k, v) in enumerate(dense(c, bt, lens)):
        ref = exact_attention(q[b], k, v, D ** -0.5 if scale is None else scale, True, window)
        check_attention(out[b], lse[b], ref, dtype, rounded, lens[b], D)
    return c, dec, dq, bt, sl, out


DECODE_CASES = [  # lengths, heads, kv heads, D, page, new, window
    ([1], 1, 1, 64, 16, 1, 0),
    ([5, 0, 16, 17, 31, 32, 33], 4, 2, 128, 16, 1, 0),
    ([127, 128, 129, 255, 257, 1], 8, 8, 64, 32, 1, 0),
    ([700, 3], 16, 1, 128, 64, 1, 0),
    ([1000], 32, 8, 128, 256, 1, 0),
    ([3, 0, 130, 2, 64], 8, 2, 128, 16, 4, 0),              # fewer tokens than new ones: rows without a key
    ([200, 90], 10, 2, 64, 128, 4, 0),                      # 20 rows: two blocks
    ([150, 33], 16, 1, 128, 16, 3, 0),                      # 48 rows: three
    ([600, 20, 129], 4, 1, 64, 64, 1, 100),
    ([600, 20, 129], 8, 2, 128, 16, 3, 1),
    ([513], 4, 4, 128, 16, 2, 130),
    ([4000], 8, 2, 128, 16, 1, 0),
]


@gpu
@pytest.mark.parametrize("dtype,kind", [(BF, BF), (HF, HF), (BF, F8), (HF, F8), (BF, I8), (HF, I8)], ids=str)
@pytest.mark.parametrize("case", DECODE_CASES, ids=str)
def test_attn_decode(case, dtype, kind):
    lens, hq, hk, D, page, new, window = case
    run_decode(lens, hq, hk, D, dtype, kind, page, new, window)


@gpu
@pytest.mark.parametrize("kind", [BF, F8], ids=str)
def test_attn_decode_widest_windows(kind):
    """Windows that reach below the first key by nearly 2^31, with fewer cached tokens than new ones."""
    for window in (2 ** 31 - 1, 2 ** 31 - 3):
        run_decode([3, 0, 130, 2, 64], 8, 2, 128, BF, kind, 16, 4, window)
        run_decode([700, 1], 4, 2, 64, BF, kind, 16, 1, window)


@gpu
def test_attn_decode_many_and_strided():
    """More sequences than a workgroup has threads, lengths of every remainder; q in a wider tensor."""
    lens = [(37 * i) % 171 for i in range(300)]
    run_decode(lens, 2, 1, 64, BF, F8, 16)
    run_decode([50, 129], 6, 3, 128, HF, I8, 32, new=2, strided=True)
    run_decode([50, 129], 6, 3, 64, BF, BF, 32, new=2, strided=True, scale=-0.3)


@gpu
@pytest.mark.parametrize("dtype,kind", [(BF, BF), (HF, HF), (BF, F8), (HF, I8)], ids=str)
def test_attn_decode_stale_pages_have_no_effect(dtype, kind):
    """What lies beyond a sequence's end in its last page, and before its window, may be NaN."""
    lens, page, window = [37, 150, 128, 401], 32, 60

    def edit(c, bt):
        for b, n in enumerate(lens):
            for part, sc in ((c.k, c.k_scale), (c.v, c.v_scale)):
                for key in list(range(n, -(-n // page) * page)) + list(range(0, max(0, n - window))):
                    p = int(bt[b, key // page])
                    if c.quantised:
                        sc[p, :, key % page] = math.nan
                        part.view(torch.uint8)[p, :, key % page] = 0x7f
                    else:
                        part[p, :, key % page] = math.nan
    run_decode(lens, 4, 2, 128, dtype, kind, page, window=window, edit=edit)

    def inside(c, bt):  # seen ones do reach the rows: the last drafted token's value, by its row alone
        p = int(bt[1, 149 // page])
        if c.quantised:
            c.v_scale[p, 0, 149 % page] = math.nan
        else:
            c.v[p, 0, 149 % page, 3] = math.inf
            c.v[p, 1, 148 % page, 5] = math.nan
    run_decode(lens, 4, 2, 128, dtype, kind, page, new=3, edit=inside)


@gpu
def test_attn_decode_faults():
    c, dec, q, bt, sl, out = run_decode([40, 40], 2, 1, 64, BF, BF, 16)
    good = bt.clone()
    for bad in (c.n_pages, -1):
        bt = good.clone()
        bt[1, 1] = bad
        got = dec(q, bt.to(DEV), sl)
        with pytest.raises(ValueError, match="block table"):
            c.check()
        assert torch.equal(got[0], out[0]) and torch.isfinite(got).all()
    for bad in (-3, 2 ** 31 - 1):
        got = dec(q, good[:, :3].contiguous().to(DEV), torch.tensor([40, bad], dtype=torch.int32, device=DEV))
        with pytest.raises(ValueError, match="lengths"):
            c.check()
        assert torch.equal(got[0], out[0])
        if bad < 0:
            assert (got[1] == 0).all()


@gpu
@pytest.mark.parametrize("dtype,kind", [(BF, BF), (HF, HF), (BF, F8), (HF, I8)], ids=str)
def test_attn_decode_bad_pages_are_not_seen(dtype, kind):
    """Keys of a page id outside the cache have no effect, whatever the cache's pages hold: the rest as without them."""
    page, lens = 16, [100, 40]
    c, dec, q, bt, sl, out = run_decode(lens, 4, 2, 64, dtype, kind, page)
    used = set(bt[0, :7].tolist()) | set(bt[1, :3].tolist())
    free = next(i for i in range(c.n_pages) if i not in used)
    if 0 in used:  # the cache's first page becomes one that no sequence names, full of NaN
        for t in (c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scale, c.v_scale):
            if t is not None:
                t[free].copy_(t[0])
        bt[bt == 0] = free
    c.k.view(torch.uint8)[0].fill_(0x7f)
    c.v.view(torch.uint8)[0].fill_(0x7f)
    if dtype != kind:
        c.k_scale[0].fill_(math.nan)
        c.v_scale[0].fill_(math.nan)
    else:
        c.k[0].fill_(math.nan)
        c.v[0].fill_(math.nan)
    assert torch.equal(dec(q, bt.to(DEV), sl), out)
    bad = bt.clone()
    bad[0, 6] = c.n_pages  # the last four keys
    got = dec(q, bad.to(DEV), sl)
    with pytest.raises(ValueError, match="block table"):
        c.check()
    k, v = dense(c, bt, lens)[0]
    # 96 keys and no mask: the last page's are those that the last token alone would have seen
    ref = exact_attention(q[0].cpu(), k[:96], v[:96], 64 ** -0.5, False, 0)
    rounded = U[dtype] if not c.quantised else U[BF] if dtype == BF else 2.0 ** -16
    check_attention(got[0], None, ref, dtype, rounded, 96, 64)
    assert torch.equal(got[1], out[1])


@gpu
def test_decode_in_a_graph_and_on_another_stream():
    """A captured step follows new contents and lengths on every replay; a call on another stream is ordered there."""
    lens = [300, 77, 5]
    c, dec, q, bt, sl, out = run_decode(lens, 8, 2, 128, BF, F8, 32)
    bt = bt.to(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert torch.equal(dec(q, bt, sl), out)
    torch.cuda.current_stream().wait_stream(side)
    static = torch.zeros_like(out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dec(q, bt, sl, out=static)
    for step in range(4):
        fill_cache(c, 50 + step)
        q.copy_(rand(*q.shape, seed=60 + step).to(DEV))
        sl.copy_(torch.tensor([300 - 90 * step, 77, 5 + 9 * step], dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        want = dec(q, bt, sl)
        torch.cuda.synchronize()
        assert torch.equal(static, want)
    c.check()


@gpu
def test_results_do_not_vary():
    """The same call twice gives the same bits: no result depends on the order in which workgroups end."""
    c, dec, q, bt, sl, out = run_decode([1500, 40, 900], 8, 1, 128, BF, BF, 16)
    for _ in range(3):
        assert torch.equal(dec(q, bt.to(DEV), sl), out)


# ------------------------------------------------------------ refusals
def lib():
    if not os.path.exists(H.library_path("release")):
        from paper_2609_40247_amd import build
        build.build()
    return O.load("release")


FAKE = 1 << 20  # an address that is only compared, never followed: every call below is refused before a launch


def fake_cache(**kw):
    a = dict(k=FAKE, v=FAKE, k_scale=None, v_scale=None, n_pages=4, n_heads=2, page_size=16, head_dim=64, kind=O.BF16)
    return O.HerschelCache(**{**a, **kw})


def st(row=128, head=64):
    return O._Strides(row, head)


def rope_args(**kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, q_strides=st(), k_strides=st(), v_strides=st(), q_out=FAKE, k_out=None,
             q_out_strides=st(), k_out_strides=st(), positions=FAKE, table=FAKE, n_positions=10, slots=FAKE, n_tokens=5,
             q_heads=2, kv_heads=2, head_dim=64, rotary_dim=64, layout=0, type=O.BF16)
    return O.HerschelRopeArgs(**{**a, **kw})


def read_args(**kw):
    a = dict(block_table=FAKE, table_stride=4, cu=FAKE, n_seqs=1, n_rows=10, k_out=FAKE, v_out=FAKE, type=O.BF16)
    return O.HerschelReadArgs(**{**a, **kw})


def prompt_args(**kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, q_strides=st(), k_strides=st(), v_strides=st(), out=FAKE, cu_q=FAKE, cu_k=FAKE,
             n_seqs=1, n_q=10, n_k=10, max_q=10, q_heads=2, kv_heads=2, head_dim=64, type=O.BF16, causal=1, scale=1.0)
    return O.HerschelPromptArgs(**{**a, **kw})


def decode_args(**kw):
    a = dict(q=FAKE, q_seq_stride=128, q_strides=st(), out=FAKE, block_table=FAKE, table_stride=4, seq_lens=FAKE,
             n_seqs=1, new_tokens=1, q_heads=2, type=O.BF16, scale=1.0, workspace=FAKE, workspace_bytes=1 << 40)
    return O.HerschelDecodeArgs(**{**a, **kw})


BAD_CACHES = [dict(k=None), dict(v=FAKE + 8), dict(n_pages=0), dict(n_heads=0), dict(page_size=24), dict(page_size=8),
              dict(page_size=512), dict(head_dim=63), dict(head_dim=258), dict(kind=4), dict(kind=O.FP8),
              dict(kind=O.INT8, k_scale=FAKE, v_scale=FAKE + 4), dict(kind=O.F16), dict(n_pages=1 << 50),
              dict(n_heads=1 << 24)]


@pytest.mark.parametrize("bad", BAD_CACHES, ids=named)
def test_bad_caches_are_refused(bad):
    c = ctypes.byref(fake_cache(**bad))
    L = lib()
    if bad.get("kind", 0) != O.F16:
        assert L.herschel_attn_decode_workspace(1, 1, 2, c, ctypes.byref(ctypes.c_size_t())) == H.EINVAL
    assert L.herschel_rope_write(ctypes.byref(rope_args()), c) == H.EINVAL
    assert L.herschel_cache_read(ctypes.byref(read_args()), c) == H.EINVAL
    assert L.herschel_attn_decode(ctypes.byref(decode_args()), c) == H.EINVAL


@pytest.mark.parametrize("bad", [
    dict(q=None, q_out=None, k=None), dict(q=None), dict(k=None), dict(v=None), dict(slots=None), dict(positions=None),
    dict(table=None), dict(table=FAKE + 4), dict(n_positions=0), dict(n_tokens=-1), dict(q_heads=0), dict(kv_heads=3),
    dict(head_dim=62, rotary_dim=62), dict(head_dim=65), dict(head_dim=0), dict(rotary_dim=66), dict(rotary_dim=31),
    dict(rotary_dim=-2), dict(layout=2), dict(type=O.FP8), dict(type=O.F16), dict(q_strides=O._Strides(-1, 64)),
    dict(k_strides=O._Strides(64, -64)), dict(q_heads=1 << 20)], ids=named)
def test_bad_rope_calls_are_refused(bad):
    assert lib().herschel_rope_write(ctypes.byref(rope_args(**bad)), ctypes.byref(fake_cache())) == H.EINVAL


@pytest.mark.parametrize("bad", [dict(n_seqs=0), dict(n_rows=-1), dict(n_rows=1 << 31), dict(table_stride=-1),
                                 dict(cu=None), dict(block_table=None), dict(k_out=FAKE + 2), dict(type=O.F16),
                                 dict(type=O.INT8)], ids=named)
def test_bad_read_calls_are_refused(bad):
    assert lib().herschel_cache_read(ctypes.byref(read_args(**bad)), ctypes.byref(fake_cache())) == H.EINVAL


@pytest.mark.parametrize("bad", [
    dict(n_seqs=0), dict(n_q=-1), dict(n_k=1 << 31), dict(max_q=-1), dict(head_dim=96), dict(kv_heads=0),
    dict(q_heads=3), dict(type=O.FP8), dict(window=-1), dict(scale=math.nan), dict(scale=math.inf), dict(cu_q=None),
    dict(cu_k=None), dict(q=None), dict(k=None), dict(out=FAKE + 4), dict(q=FAKE + 1),
    dict(v_strides=O._Strides(-1, 0))], ids=named)
def test_bad_prompt_calls_are_refused(bad):
    assert lib().herschel_attn_prompt(ctypes.byref(prompt_args(**bad))) == H.EINVAL


@pytest.mark.parametrize("bad,code", [
    (dict(n_seqs=0), H.EINVAL), (dict(n_seqs=4097), H.EINVAL), (dict(new_tokens=0), H.EINVAL), (dict(q_heads=3), H.EINVAL),
    (dict(q=None), H.EINVAL), (dict(out=FAKE + 8), H.EINVAL), (dict(seq_lens=None), H.EINVAL),
    (dict(block_table=None), H.EINVAL), (dict(table_stride=-1), H.EINVAL), (dict(type=O.F16), H.EINVAL),
    (dict(window=-1), H.EINVAL), (dict(scale=math.nan), H.EINVAL), (dict(q_seq_stride=-1), H.EINVAL),
    (dict(workspace=None), H.EWORKSPACE), (dict(workspace=FAKE + 128), H.EWORKSPACE),
    (dict(workspace_bytes=1000), H.EWORKSPACE)], ids=named)
def test_bad_decode_calls_are_refused(bad, code):
    assert lib().herschel_attn_decode(ctypes.byref(decode_args(**bad)), ctypes.byref(fake_cache())) == code


def test_null_arguments_are_refused():
    L = lib()
    assert L.herschel_rope_write(None, None) == H.EINVAL
    assert L.herschel_cache_read(ctypes.byref(read_args()), None) == H.EINVAL
    assert L.herschel_attn_prompt(None) == H.EINVAL
    assert L.herschel_attn_decode(ctypes.byref(decode_args()), None) == H.EINVAL
    assert L.herschel_attn_decode_workspace(1, 1, 2, ctypes.byref(fake_cache()), None) == H.EINVAL
    # nothing to do is not an error
    assert L.herschel_rope_write(ctypes.byref(rope_args(n_tokens=0)), ctypes.byref(fake_cache())) == H.OK
    assert L.herschel_cache_read(ctypes.byref(read_args(n_rows=0)), ctypes.byref(fake_cache())) == H.OK
    assert L.herschel_attn_prompt(ctypes.byref(prompt_args(n_q=0, max_q=0))) == H.OK


def test_operator_struct_layouts_match_the_header(tmp_path):
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = {"herschel_cache": O.HerschelCache, "herschel_rope_args": O.HerschelRopeArgs,
               "herschel_read_args": O.HerschelReadArgs, "herschel_prompt_args": O.HerschelPromptArgs,
               "herschel_decode_args": O.HerschelDecodeArgs, "herschel_strides": O._Strides}
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "herschel_ops.h"', "int main(void) {"]
    for cname, cls in structs.items():
        lines.append(f'  printf("{cname} %zu\\n", sizeof({cname}));')
        lines += [f'  printf("{cname}.{f} %zu\\n", offsetof({cname}, {f}));' for f, _ in cls._fields_]
    (tmp_path / "layout.c").write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    exe = str(tmp_path / "layout")
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(root, "include"), "-o", exe, str(tmp_path / "layout.c")], check=True)
    got = dict(line.split() for line in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines())
    for cname, cls in structs.items():
        assert int(got[cname]) == ctypes.sizeof(cls), cname
        for f, _ in cls._fields_:
            assert int(got[f"{cname}.{f}"]) == getattr(cls, f).offset, f"{cname}.{f}"


def test_packed_arguments_match_the_structures():
    """The formats that calls are packed with lay every field where the ctypes structure has it."""
    for fmt, cls in ((O._ROPE, O.HerschelRopeArgs), (O._READ, O.HerschelReadArgs), (O._PROMPT, O.HerschelPromptArgs),
                     (O._DECODE, O.HerschelDecodeArgs)):
        flat = []
        for name, kind in cls._fields_:
            flat += [(name, f) for f, _ in kind._fields_] if hasattr(kind, "_fields_") else [(name, None)]
        assert fmt.size <= ctypes.sizeof(cls)
        got = cls.from_buffer_copy(fmt.pack(*range(1, len(flat) + 1)).ljust(ctypes.sizeof(cls), b"\0"))
        for i, (name, part) in enumerate(flat):
            x = getattr(got, name)
            assert (getattr(x, part) if part else x) == i + 1, (cls.__name__, name)


def test_tensor_checks_on_the_cpu():
    """The binding refuses tensors that are not on a GPU, or of the wrong kind, before it calls the library."""
    x = torch.zeros(4, 2, 64, dtype=BF)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        O.attn_prompt(x, x, x, i, max_q=4)
    with pytest.raises(ValueError, match="GPU"):
        O.rope_write(x, None, None, torch.zeros(4, dtype=torch.int64), torch.zeros(9, 32, 2))
    with pytest.raises(ValueError):
        O.PagedCache(torch.zeros(1, 1, 16, 64), torch.zeros(1, 1, 16, 64))
    with pytest.raises(ValueError, match="q or k"):
        O.rope_write(None, None, None, i, x)


@gpu
def test_tensor_checks():
    x = torch.zeros(4, 2, 64, dtype=BF, device=DEV)
    cu = torch.tensor([0, 4], dtype=torch.int32, device=DEV)
    for kw in (dict(k=x.to(HF)), dict(k=x[:, :, :32]), dict(cu_q=cu.long()), dict(cu_q=cu.cpu()), dict(max_q=5),
               dict(window=-1), dict(k=x[:, :0]), dict(q=x.transpose(1, 2)), dict(q=x[0]), dict(out=x[:2]),
               dict(status=torch.zeros(2, dtype=torch.int32, device=DEV)), dict(q=x.float())):
        a = {**dict(q=x, k=x, v=x, cu_q=cu, max_q=4), **kw}
        with pytest.raises(ValueError):
            O.attn_prompt(a.pop("q"), a.pop("k"), a.pop("v"), a.pop("cu_q"), **a)
    c = O.PagedCache.allocate(2, 2, 16, 64, BF, DEV)
    pos, table = torch.zeros(4, dtype=torch.int64, device=DEV), O.rotary_table(5, 64, device=DEV)
    for kw in (dict(slots=None), dict(slots=pos.int()), dict(positions=pos[:2]), dict(table=table.half()), dict(v=x[:2]),
               dict(layout="other"), dict(k=x[:, :1], v=x[:, :1]), dict(q=x.to(HF), k=x.to(HF), v=x.to(HF)),
               dict(q_out=x[:, :1]), dict(v=None)):
        a = {**dict(q=x, k=x, v=x, positions=pos, table=table, cache=c, slots=pos), **kw}
        with pytest.raises(ValueError):
            O.rope_write(a.pop("q"), a.pop("k"), a.pop("v"), a.pop("positions"), a.pop("table"), **a)
    bt = torch.zeros(1, 2, dtype=torch.int32, device=DEV)
    for kw in (dict(cu=cu.long()), dict(block_table=bt.long()), dict(block_table=bt[0]), dict(total=-1), dict(dtype=HF),
               dict(block_table=torch.cat([bt, bt])), dict(k_out=x[:1])):
        a = {**dict(block_table=bt, cu=cu, total=4), **kw}
        with pytest.raises(ValueError):
            O.cache_read(c, a.pop("block_table"), a.pop("cu"), **a)
    dec = O.DecodeAttention(c, batch=1, heads=4)
    q = torch.zeros(1, 1, 4, 64, dtype=BF, device=DEV)
    n = torch.zeros(1, dtype=torch.int32, device=DEV)
    for kw in (dict(q=q[:, :, :2]), dict(q=q.to(HF)), dict(q=torch.cat([q, q])), dict(seq_lens=n.long()),
               dict(block_table=bt.cpu()), dict(window=-1), dict(out=q[0])):
        a = {**dict(q=q, block_table=bt, seq_lens=n), **kw}
        with pytest.raises(ValueError):
            dec(a.pop("q"), a.pop("block_table"), a.pop("seq_lens"), **a)
    for kw in (dict(batch=0), dict(heads=3), dict(new_tokens=0), dict(dtype=HF), dict(batch=5000)):
        with pytest.raises(ValueError):
            O.DecodeAttention(c, **{**dict(batch=1, heads=4), **kw})


# ------------------------------------------------------------ the operators together
@gpu
@pytest.mark.parametrize("cache", ["bf16", "fp8", "int8"])
def test_layer_prompt_and_steps_agree(cache):
    """A token attended to in a decode step and the same token as a prompt's last: one computes from the cache what the
    other computes from its rows; with a 16-bit cache both stay within their bounds of the 64-bit result, with codes
    they differ by what the codes round away."""
    from paper_2609_40247_amd import reference as R
    lens, D, h, g = [40, 130, 1, 77], 64, 4, 2
    total = [n + 1 for n in lens]
    x = [rand(n, h + 2 * g, D, seed=90 + i) for i, n in enumerate(total)]
    whole, parts = (R.AttentionLayer(h, g, D, len(lens), 200, 16, cache) for _ in range(2))
    a = whole.prompt(torch.cat(x).to(DEV), total)
    parts.prompt(torch.cat([t[:-1] for t in x]).to(DEV), lens)
    b = parts.step(torch.stack([t[-1] for t in x]).to(DEV))
    whole.cache.check(), parts.cache.check()
    assert parts.lengths.tolist() == total
    last = torch.tensor(total).cumsum(0) - 1
    for i, n in enumerate(total):
        k = exact_rope(x[i][:, h:h + g], whole.table.cpu()[:n], "half", D)[0].to(BF)
        q = exact_rope(x[i][:, :h], whole.table.cpu()[:n], "half", D)[0].to(BF)
        ref = exact_attention(q[-1:], k, x[i][:, h + g:], D ** -0.5, True, 0)
        # the rotation's own rounding to bf16 may fall the other way in 32 bits: one more unit of each product
        o, lse, A, S = ref
        slack = 2 * 2.0 ** -8 * (A + S[..., None] * A)
        assert ((a[last[i]].double().cpu() - o[0]).abs() <= U[BF] * o[0].abs() + 2 * U[BF] * A[0] + slack[0]).all()
        step = {"bf16": 0.0, "fp8": 2.0 ** -4, "int8": 0.5 / 127 * 4}[cache]  # of a row's elements (int8: peak over rms)
        coarse = step * (A + 2 * S[..., None] * A)
        assert ((b[i].double().cpu() - o[0]).abs() <= U[BF] * o[0].abs() + 2 * U[BF] * A[0] + slack[0] + coarse[0]).all()


@gpu
def test_reference_sol():
    """The command's figures are the analyzer's own, and the trace that it rates is the calls'."""
    import oracle
    from paper_2609_40247_amd import reference as R
    r = R.reference_sol(heads=8, kv_heads=2, head_dim=64, prompt=300, batch=3, prompts=2, steps=4, cache="int8", page_size=32)
    assert list(r["ops"]) == list(R.OPS)
    assert [o["calls"] for o in r["ops"].values()] == [1, 1, 4, 4]
    for o in r["ops"].values():
        assert o["ns"] > 0 and o["sol"] == max(o["mfu"], o["mbu"]) > 0
    code, want = oracle.analyze(r["columns"], r["params"], gap_capacity=100)
    assert code == 0
    for k in ("op_sol", "opn_sol", "opn_time", "opn_flops", "opn_bytes"):
        assert (want[k] == r["outputs"][k]).all(), k


def test_counts_of_the_layer():
    """Operations and bytes of a decode step are those of the paged-attention case: 36 layers of 32 and 8 heads of
    128 over 4000 tokens are 2.36 GFLOP and 0.59 GB."""
    from types import SimpleNamespace

    from paper_2609_40247_amd import reference as R
    layer = SimpleNamespace(heads=32, kv_heads=8, head_dim=128,
                            cache=SimpleNamespace(k=torch.zeros(1, dtype=BF), quantised=False))
    f, b = R.counts(layer, "attn_decode", [4000])
    assert round(36 * f / 1e9, 2) == 2.36 and round(36 * b / 1e9, 2) == 0.59
    f, b = R.counts(layer, "attn_prompt", [3])
    assert f == 4 * 128 * 32 * 6 and b == 3 * 80 * 256
    f, b = R.counts(layer, "rope_write_step", [5, 9])
    assert f == 3 * 2 * 40 * 128 and b == 2 * (80 * 256 + 16 * 256 + 512 + 16)


@gpu
def test_windows_beyond_32_bits_are_refused():
    x = rand(4, 2, 64).to(DEV)
    cu = torch.tensor([0, 4], dtype=torch.int32, device=DEV)
    c = make_cache(BF, 2, 2, 16, 64)
    dec = O.DecodeAttention(c, batch=1, heads=2)
    with pytest.raises(ValueError, match="window"):
        O.attn_prompt(x, x, x, cu, max_q=4, window=2 ** 31)
    with pytest.raises(ValueError, match="window"):
        dec(x[None, :1], torch.zeros(1, 2, dtype=torch.int32, device=DEV), cu[:1], window=2 ** 31)
