"""The operators around the attention at sizes, strides and memory where a call
goes another way than its neighbours.  Tolerances are those of
``test_layer_operators``, derived there."""
from __future__ import annotations

import json
import random

import pytest
import torch

from paper_2609_40247_amd import operators as O
from test_host_calls import child, fake  # noqa: F401
from test_layer_operators import BF, DEV, F8, HF, I8, check_product, device_weights, gpu, make_rows8, make_weights, rand


# Calls over the stand-in for the HIP runtime: what is launched, on a machine without a GPU.
PRODUCT = '''
import struct
device()
BF16, F16, FP8, INT8 = 0, 1, 2, 3

def product(rows, n, k, group, kind=BF16, x_group=0, gated=0, workspace=0, x=1 << 40, x_row=None, out=1 << 50, x_scale=1 << 51,
            codes=1 << 52, scales=1 << 53):
    w = struct.pack("@2P3i", codes, scales, n, k, group)
    a = struct.pack("@Pq2Pq4iPNP", x, k if x_row is None else x_row, x_scale if kind > 1 else 0, out, rows, kind, x_group,
                    0 if kind > 1 else kind, gated, 1 << 54 if workspace else 0, workspace, 0)
    code = lib.herschel_product4(a, w)
    return code, [line.split()[1:8] for line in log() if line.startswith("launch ")]  # name, grid, threads, "lds", bytes
'''


NORM = '''
import struct
device()
BF16, F16, FP8, INT8, F32 = 0, 1, 2, 3, 4

def norm(n, dim, x, x_row, out, residual=0, residual_row=0, kept=0, kept_row=0, weight=1 << 40, scale=0, group=0, residual_type=BF16,
         weight_type=BF16, kind=BF16):
    a = struct.pack("@PqPqPq3Pq6ifP", x, x_row, residual, residual_row, kept, kept_row, weight, out, scale, n, dim, group, BF16,
                    residual_type, weight_type, kind, 1e-6, 0)
    code = lib.herschel_norm_rows(a)
    return code, sum(line.startswith("launch ") for line in log())
'''


# ------------------------------------------------------------ products of 8-bit rows with a scale for each group
def test_phases_of_rows_begin_where_their_addresses_say(fake):  # noqa: F811
    """Addresses in a phase of x are made with exclusive ors below 128 bytes, so each phase begins at a multiple of 128,
    with odd numbers of rows and their scales too, and several of them are that many bytes in all."""
    sizes = child(fake, PRODUCT + '''
for rows in range(1, 66):
    for k in (256, 1024, 1152, 2048, 5120, 25_600):
        for group in (32, 64, 128):
            code, launched = product(rows, 96, k, group, INT8, x_group=group)
            out.append((code, [int(line[6]) for line in launched]))
''')
    assert all(code == 0 and len(lds) == 1 and lds[0] % 128 == 0 for code, lds in sizes)


def group_rows(rows, k, kind, group, seed):
    """8-bit rows with a scale for each group of columns, of which the last may have fewer, on the GPU; their values in
    64 bits."""
    groups = -(-k // group)
    x = torch.nn.functional.pad(rand(rows, k, seed=seed), (0, groups * group - k))
    # groups of different magnitudes, so that no scale can stand for another
    x = x.float() * (2.0 ** (torch.arange(groups) % 5)).repeat_interleave(group)
    r = make_rows8(x, kind, group)
    wide = (r.codes.double() * r.scale.double().repeat_interleave(group, 1))[:, :k]
    return O.Rows8(r.codes[:, :k].contiguous().to(DEV), r.scale.to(DEV)), wide


@gpu
@pytest.mark.parametrize("kind", [F8, I8], ids=str)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows", [1, 3, 16, 17, 31, 32, 33, 63, 64, 65, 97, 129])
def test_product4_of_rows_with_group_scales(rows, group, kind):
    """Even and odd numbers of rows, of one to many phases of columns, gated and not; the last group whole and not."""
    for k in (1024, 1088, 2048, 5120, 1500):
        codes, scales, zero, w, size = make_weights(96, k, group, True, seed=k)
        W = device_weights(codes, scales, zero, k)
        r, wide = group_rows(rows, k, kind, group, rows)
        assert torch.equal(r.values().cpu(), wide.float())
        for gated in (False, True):
            check_product(O.product4(r, W, gated=gated), wide, w, size, group, BF, gated)


@gpu
@pytest.mark.parametrize("kind", [F8, I8], ids=str)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,n,k", [(5, 8400, 2112), (21, 8320, 2048), (33, 4224, 1088), (47, 8448, 2048), (131, 4176, 1984),
                                      (35, 48, 15_040), (19, 64, 16_400), (3, 70, 20_032)])
def test_product4_of_rows_with_group_scales_in_wide_workgroups_and_parts(rows, n, k, group, kind):
    """Many weight rows, whose workgroups are wider, and few with long columns, which several workgroups share."""
    codes, scales, zero, w, size = make_weights(n, k, group, True, HF, seed=n)
    r, wide = group_rows(rows, k, kind, group, k)
    check_product(O.product4(r, device_weights(codes, scales, zero, k), dtype=HF), wide, w, size, group, HF)


# ------------------------------------------------------------ workspaces
def test_product4_shares_columns_only_where_the_workspace_says(fake):  # noqa: F811
    """A workspace with room for more is used as the size that is asked for says: not at all beyond 4096 rows, whose
    parts one launch could not join."""
    sizes = child(fake, PRODUCT + """
size = ctypes.c_size_t(0)
for rows in (1, 64, 1000, 4096, 4097, 65_535, 65_536, 70_000, 4_194_240):
    for n, k, gated in ((16, 25_600, 0), (64, 25_600, 1), (640, 128_000, 0), (16, 100, 0)):
        assert lib.herschel_product4_workspace(ctypes.c_int64(rows), BF16, gated, n, k, ctypes.byref(size)) == 0
        code, launched = product(rows, n, k, 128, gated=gated, workspace=1 << 50)
        out.append((code, rows, size.value // (rows * -(-n // 16) * 64), [[int(v) for v in line[1:4]] for line in launched]))
""")
    assert {parts > 0 for code, rows, parts, _ in sizes if rows <= 4096} == {True, False}
    for code, rows, parts, launched in sizes:
        assert code == 0 and (parts == 0 or rows <= 4096)
        assert len(launched) == (2 if parts else 1) and launched[0][2] == max(1, parts)
        assert all(y <= 65_535 for _, y, _ in launched)


@gpu
def test_product4_of_many_rows_leaves_a_workspace_alone():
    rows, n, k, group = 70_000, 16, 25_600, 128
    codes, scales, zero, w, size = make_weights(n, k, group, True)
    W = device_weights(codes, scales, zero, k)
    x = rand(k + 8 * (rows - 1), seed=3)
    given = x.to(DEV).as_strided((rows, k), (8, 1))  # each row 8 elements behind the one before
    want = O.product4(given, W)
    some = [0, 1, 4095, 4096, 65_535, 65_536, rows - 1]
    check_product(want[some], torch.stack([x[8 * i:8 * i + k] for i in some]).double(), w, size, group, BF)
    workspace = torch.full((4 * rows * 16,), 7.0, device=DEV)
    out = torch.empty_like(want)
    args = O._PRODUCT.pack(given.data_ptr(), 8, 0, out.data_ptr(), rows, O.BF16, 0, O.BF16, 0, workspace.data_ptr(),
                           workspace.numel() * 4, torch.cuda.current_stream().cuda_stream)
    assert O.load().herschel_product4(args, W._at) == 0
    assert torch.equal(out, want) and (workspace == 7).all()


# ------------------------------------------------------------ what is written over what is read
def norm_memory(rng):
    """A small norm call with its tensors close together, and whether it is to be refused: from the bytes of each."""
    n, dim = rng.choice([1, 2, 3, 7]), rng.choice([1, 2, 5, 32])
    kind = rng.choice([0, 0, 0, 2, 3])
    group = 32 if kind and dim == 32 and rng.random() < 0.5 else 0
    residual_type = rng.choice([0, 0, 4]) if rng.random() < 0.7 else None
    e = 4 if residual_type == 4 else 2
    base = 1 << 20
    room = rng.choice([200, 1000, 8000])

    def at(align):
        return base + rng.randrange(room) // align * align
    steps = [dim, dim + 1, dim + 8, 2 * dim, 3 * dim, 100]
    c = dict(n=n, dim=dim, x=at(2), x_row=rng.choice([0, 1] + steps), out=at(1 if kind else 2), weight=at(4), kind=kind, group=group,
             weight_type=rng.choice([0, 4]), scale=at(4) if kind else 0)
    if residual_type is not None:
        c.update(residual=at(e), residual_row=rng.choice([0, 1] + steps), residual_type=residual_type)
        if rng.random() < 0.8:
            c.update(kept=at(e), kept_row=rng.choice(steps))
    # the same rows, now and then
    if rng.random() < 0.3:
        c.update(out=c["x"], x_row=rng.choice([dim, c["x_row"]]))
    if "kept" in c and rng.random() < 0.4:
        c.update(residual=c["kept"], residual_row=rng.choice([c["kept_row"], c["residual_row"]]))
    elif "kept" in c and e == 2 and rng.random() < 0.4:
        c.update(x=c["kept"], x_row=rng.choice([c["kept_row"], c["x_row"]]))

    def rows(start, step, width, size):
        return [range(start + r * step * size, start + (r * step + width) * size) for r in range(n)]
    read = dict(x=rows(c["x"], c["x_row"], dim, 2), weight=[range(c["weight"], c["weight"] + dim * (4 if c["weight_type"] else 2))])
    written = dict(out=rows(c["out"], dim, dim, 1 if kind else 2))
    if kind:
        groups = dim // group if group else 1
        written["scale"] = rows(c["scale"], groups, groups, 4)
    if "residual" in c:
        read["residual"] = rows(c["residual"], c["residual_row"], dim, e)
    if "kept" in c:
        written["kept"] = rows(c["kept"], c["kept_row"], dim, e)
    sets = {k: {b for r in v for b in r} for k, v in {**read, **written}.items()}
    bad = False
    for w in written:
        for o in [*read, *written]:
            same = (w, o) in (("kept", "residual"), ("kept", "x"), ("out", "x")) and written[w] == read[o]
            bad |= w != o and not same and bool(sets[w] & sets[o])
    return c, bad


def test_norm_rows_over_other_rows_are_refused(fake, tmp_path):  # noqa: F811
    """What is written may be the rows that it stands for; any other byte that it shares with what is read, or written
    as well, would be read before or after it changes.  Rows between another tensor's rows are none."""
    rng = random.Random(1)
    cases = [norm_memory(rng) for _ in range(6000)]
    (tmp_path / "cases.json").write_text(json.dumps([c for c, _ in cases]))
    codes = child(fake, NORM + f"out += [norm(**c) for c in json.load(open({str(tmp_path / 'cases.json')!r}))]\n")
    bad = [b for _, b in cases]
    assert 500 < sum(bad) < 5500 and codes == [[-1, 0] if b else [0, 1] for b in bad]


def test_norm_rows_beside_other_rows(fake):  # noqa: F811
    """Tensors that are columns of one buffer, of many rows: shifted by an element they are refused."""
    codes = child(fake, NORM + """
n, dim, X = 2_000_000, 64, 1 << 30
for shift in (0, 128, 130, 126, -128, -126, 256, 258):
    for step in (192, 191, 193, 384, 100):  # of the residual's rows; those of x lie 192 elements apart
        out.append((shift, step, norm(n, dim, X, 192, 1 << 50, X + shift, step, X + shift, step)[0]))
out.append((0, 0, norm(n, dim, X, dim, X)[0]))
out.append((2, 0, norm(n, dim, X, dim, X + 2)[0]))
out.append((2, 0, norm(n, dim, X, dim, X + n * dim * 2 - 2)[0]))
out.append((0, 0, norm(n, dim, X, dim, X + n * dim * 2)[0]))
""")
    for shift, step, code in codes:
        # x's rows take 128 of every 384 bytes; those of the residual fit between them if they keep their place in it
        between = step in (192, 384) and 128 <= shift % 384 <= 256
        fine = shift == 0 if step == 0 else between or (step, shift) == (192, 0)
        assert (code == 0) == fine, (shift, step)


@gpu
def test_norm_rows_in_shared_buffers():
    """Rows, sums and residual as columns of one buffer, and a residual stream that is the rows; shifted ones are refused."""
    n, dim = 37, 264
    big, w = rand(n, 3 * dim, seed=1, dtype=HF).to(DEV), rand(dim, seed=2, dtype=HF).to(DEV)
    x, r, kept = big[:, :dim], big[:, dim:2 * dim], big[:, 2 * dim:]
    sums = torch.empty(n, dim, dtype=HF, device=DEV)
    want = O.norm_rows(x.clone(), w, r.clone(), residual_out=sums)
    before = big.clone()
    assert torch.equal(O.norm_rows(x, w, r, residual_out=kept), want)
    assert torch.equal(kept, sums) and torch.equal(big[:, :2 * dim], before[:, :2 * dim])
    assert torch.equal(O.norm_rows(x, w, r, residual_out=x), want) and torch.equal(x, sums)
    twice = O.norm_rows(r.clone(), w, r.clone())
    assert torch.equal(O.norm_rows(r, w, r), twice)  # a stream that is the rows
    before = big.clone()
    line = big.view(-1)
    for bad in (dict(residual=r, residual_out=big[:, 1:dim + 1]), dict(residual=r, residual_out=big[:, dim + 1:2 * dim + 1]),
                dict(out=line[:n * dim].view(n, dim)), dict(residual=x, out=line[2 * dim + 1:][:n * dim].view(n, dim)),
                dict(kind=I8, out=O.Rows8(line.view(I8)[:n * dim].view(n, dim), torch.empty(n, 1, device=DEV))),
                dict(x=line[:n * dim].view(n, dim), out=line[1:n * dim + 1].view(n, dim)),
                dict(x=line[:n * dim].view(n, dim), residual=r.clone(), out=line[:n * dim].view(n, dim), residual_out=line[:n * dim].view(n, dim)),
                dict(weight=line[:dim], x=r, out=line[:n * dim].view(n, dim))):
        with pytest.raises(ValueError):
            O.norm_rows(**{**dict(x=x, weight=w), **bad})
    assert torch.equal(big, before)


def test_product4_over_what_it_reads_is_refused(fake):  # noqa: F811
    """An output over rows, their scales or the weights; between rows that lie far apart there is room for one."""
    codes = child(fake, PRODUCT + """
X, rows, n, k = 1 << 40, 5, 48, 256  # an output of 480 bytes, rows of 512 (8 bits: 256), 6 KB of codes, 48 x 2 words of scales
for kind, e in ((BF16, 2), (INT8, 1)):
    for x_row in (k, 1024):
        for at in range(-600, 6000, 2):
            out.append((kind, at, [(r * x_row * e, r * x_row * e + k * e) for r in range(rows)],
                        product(rows, n, k, 128, kind, x_row=x_row, x=X, out=X + at)[0]))
S = 1 << 51
for at in range(-600, 200, 2):
    out.append((INT8, at, [(0, rows * 2 * 4)], product(rows, n, k, 128, INT8, x_group=128, x_scale=S, out=S + at)[0]))
for at in range(-600, 6800, 2):
    out.append((BF16, at, [(0, 6144)], product(rows, n, k, 128, codes=S, out=S + at)[0]))
    out.append((BF16, at, [(0, 48 * 2 * 4)], product(rows, n, k, 128, scales=S, out=S + at)[0]))
""")
    refused = 0
    for kind, at, read, code in codes:
        over = any(a < at + 480 and at < b for a, b in read)
        assert code == (-1 if over else 0), (kind, at, read)
        refused += over
    assert 1000 < refused < len(codes) - 1000


@gpu
def test_product4_between_rows():
    """An output that lies between rows of x, which it leaves alone."""
    codes, scales, zero, w, size = make_weights(48, 256, 64, True)
    W = device_weights(codes, scales, zero, 256)
    big = rand(5, 1024, seed=8).to(DEV)
    before = big.clone()
    out = big[2, 300:300 + 5 * 48].view(5, 48)
    check_product(O.product4(big[:, :256], W, out=out), before[:, :256].cpu().double(), w, size, 64, BF)
    before[2, 300:540] = big[2, 300:540]
    assert torch.equal(big, before)


def test_verify_drafts_over_what_it_reads_is_refused(fake):  # noqa: F811
    """Tokens, counts and workspaces over the inputs, or over one another; between rows of probabilities there is room."""
    codes = child(fake, """
import struct
device()
B, S = 3, 2
A = {k: 1 << 40 + i for i, k in enumerate(("target", "draft", "tokens", "counts", "accept_u", "final_u", "out", "accepted", "workspace"))}

def verify(vocab, drafted=True, **at):
    a = {**A, **at}
    row = 40_000
    args = struct.pack("@P2qP2q6P4iPN2P", a["target"], (S + 1) * row, row, a["draft"] if drafted else 0, S * row, row, a["tokens"],
                       a["counts"], a["accept_u"], a["final_u"], a["out"], a["accepted"], B, S, vocab, 4, a["workspace"], 1 << 30, 0, 0)
    code = lib.herschel_verify_drafts(args)
    return code, sum(line.startswith("launch ") for line in log())

need = ctypes.c_size_t(0)
assert lib.herschel_verify_workspace(B, 39_000, ctypes.byref(need)) == 0
spans = {v: dict(target=[(r * 160_000, v * 4) for r in range(B * (S + 1))], draft=[(r * 160_000, v * 4) for r in range(B * S)],
                 tokens=[(0, B * S * 8)], counts=[(0, B * 4)], accept_u=[(0, B * S * 4)], final_u=[(0, B * 4)],
                 out=[(0, B * (S + 1) * 8)], accepted=[(0, B * 4)], workspace=[(0, need.value if v > 32_768 else 0)]) for v in (39_000, 1000)}
for v, of in spans.items():
    for w in ("out", "accepted", "workspace"):
        size = of[w][0][1]
        for other in A:
            if w == other or not size or not of[other][0][1]:
                continue
            for begin, n in of[other]:
                for shift, bad in ((-size, False), (16 - size, True), (0, True), ((n + 15) // 16 * 16 - 16, True), ((n + 15) // 16 * 16, False)):
                    out.append((v, w, other, begin + shift, bad, verify(v, **{w: A[other] + begin + shift})))
out.append((1000, "", "", 0, False, verify(1000)))
out.append((1000, "out", "draft", 0, False, verify(1000, drafted=False, out=A["draft"])))
""")
    assert len(codes) > 200
    for *case, bad, (code, launched) in codes:
        if case[1] == "workspace" and case[3] % 16:
            assert code == -4 and not launched, case  # that it is not aligned is found first
        else:
            assert (code, launched) == ((-1, 0) if bad else (0, 2 if case[0] > 32_768 else 1)), case


# ------------------------------------------------------------ 8-bit rows as numbers
@pytest.mark.parametrize("columns,group", [(200, 64), (1500, 128), (1500, 64), (1500, 32), (96, 32), (64, 64), (130, 128), (40, 32),
                                           (512, 64), (7, 0), (200, 0), (512, 256)])
def test_rows8_values_of_a_shorter_last_group(columns, group):
    """The groups are those that a product takes the scales for: of 32, 64 or 128 columns, the last with what is left."""
    r = O.Rows8(rand(3, columns, seed=1, gain=40.0).to(I8), 2.0 ** (torch.arange(3 * -(-columns // (group or columns))) % 11 - 5.0).view(3, -1))
    want = torch.empty(3, columns)
    for j in range(columns):
        want[:, j] = r.codes[:, j].float() * r.scale[:, j // (group or columns)]
    assert torch.equal(r.values(), want)


def test_rows8_values_of_scales_that_fit_no_group():
    with pytest.raises(ValueError, match="scale"):
        O.Rows8(torch.zeros(3, 200, dtype=I8), torch.ones(3, 3)).values()


@gpu
def test_norm_rows_refuses_scales_that_require_gradients():
    """An output of 8-bit rows whose scales are a leaf would be cut off from the rows without a word, as any other."""
    x, w = rand(4, 64).to(DEV), rand(64).to(DEV)
    out = O.Rows8(torch.zeros(4, 64, dtype=I8, device=DEV), torch.zeros(4, 1, device=DEV, requires_grad=True))
    with pytest.raises(ValueError, match="no backward"):
        O.norm_rows(x, w, kind=I8, out=out)
    with torch.no_grad():
        O.norm_rows(x, w, kind=I8, out=out)
    assert torch.equal(out.scale.detach(), O.norm_rows(x, w, kind=I8).scale)


# ------------------------------------------------------------ the largest
def test_product4_launches_of_the_most_weight_rows(fake):  # noqa: F811
    """A launch's threads are counted in 32 bits along each line of workgroups: matrices are taken up to the last one
    whose launch they hold."""
    most = 715_827_840
    assert O.MAX_WEIGHT_ROWS == most
    calls = child(fake, PRODUCT + f"""
size = ctypes.c_size_t(0)
for n in ({most}, {most} - 31, {most} // 64 * 32, 1 << 29, 1 << 28, 1 << 27, 10 ** 8, 1 << 24):
    for rows in (1, 16, 17, 64, 65, 4_194_240):
        for k in (1, 1024, 50_000, 1 << 30):
            for kind, gated in ((BF16, 0), (INT8, 0), (FP8, 1)):
                if not gated or n % 32 == 0:
                    out.append(product(rows, n, k, 128, kind, gated=gated, out=1 << 61, x=1 << 40, codes=1 << 60, scales=1 << 60, x_row=0))
                    assert lib.herschel_product4_workspace(ctypes.c_int64(rows), kind, gated, n, k, ctypes.byref(size)) == 0
out.append((product(1, {most} + 1, 1, 128)[0], None))
out.append((lib.herschel_product4_workspace(ctypes.c_int64(1), 0, 0, {most} + 1, 1, ctypes.byref(size)), None))
""")
    assert [code for code, launched in calls if launched is None] == [-1, -1]
    for code, launched in calls[:-2]:
        assert code == 0 and len(launched) == 1
        x, y, z, threads = (int(v) for v in launched[0][1:5])
        assert x * threads < 1 << 32 and max(y, z) <= 65_535
    with pytest.raises(ValueError, match="at most"):
        O.Weights4(torch.zeros(1, 1, dtype=torch.uint8).expand(most + 1, 1), torch.zeros(1, 1, dtype=BF).expand(most + 1, 1))
