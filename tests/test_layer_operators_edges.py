"""The operators around the attention at sizes, strides and memory where a call
goes another way than its neighbours.  Tolerances are those of
``test_layer_operators``, derived there."""
from __future__ import annotations

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
