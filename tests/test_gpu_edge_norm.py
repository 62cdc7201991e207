"""jdob_edge_norm against its definition in 64 bits."""

import pytest
import torch

from paper_2504_14611_amd import edge
from tests import edge_model as model

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def inputs(rows, dim, dtype, residual, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, dim, generator=gen, device="cuda").to(dtype)
    r = torch.randn(rows, dim, generator=gen, device="cuda").mul_(3).to(dtype) if residual else None
    w = torch.randn(dim, generator=gen, device="cuda").add_(1).to(dtype)
    return x, r, w


def check(r, x, w, eps, residual, label):
    h, y = model.norm(x, w, eps, residual)
    if residual is not None:
        assert torch.equal(r["sum"], (x.float() + residual.float()).to(x.dtype)), label
    if r["out"] is not None:
        off = (r["out"].double() - y).abs() - model.norm_bound(y, x.dtype)
        assert off.max() <= 0, (label, off.max())
    if r["q"] is not None:
        top = y.abs().amax(dim=1)
        assert ((r["scale"].double() - top / 127).abs() <= top / 127 * 100 * model.U32).all(), label
        step = torch.where(top > 0, top / 127, 1.0)[:, None]
        # the nearest integer, or its neighbour where y / step lies at the middle to 127 roundings of 100 steps
        assert ((r["q"].double() - y / step).abs() <= 0.5 + 127 * 101 * model.U32).all(), label
        assert (r["q"].abs().amax(dim=1)[top > 0] == 127).all(), label


@pytest.mark.parametrize("dtype", [BF16, F16, F32], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,dim", [(1, 1), (1, 4096), (3, 7), (5, 64), (2, 513), (33, 1000), (1025, 1031),
                                      (1500, 512), (1024, 2048), (1030, 4096), (7, 8192), (3, 16384), (2, 12345)])
def test_norm(rows, dim, dtype):
    for residual in (False, True):
        x, r, w = inputs(rows, dim, dtype, residual, rows + dim)
        for bits8, out16 in ((False, True), (True, False), (True, True)):
            got = edge.norm(x, w, eps=1e-5, residual=r, bits8=bits8, out16=out16)
            check(got, x, w, 1e-5, r, (rows, dim, dtype, residual, bits8, out16))


@pytest.mark.parametrize("shift", [0, 1, 3])
def test_norm_strides_offsets_and_in_place(shift):
    """Rows that start at any element, wider strides, and the sum written over the residual or over x."""
    rows, dim = 1100, 1024
    gen = torch.Generator(device="cuda").manual_seed(1)
    wide = torch.randn(rows, dim + 40, generator=gen, device="cuda").to(BF16)
    x, (_, r, w) = wide[:, shift:shift + dim], inputs(rows, dim, BF16, True)
    qs = torch.full((rows, dim + 24), 99, dtype=torch.int8, device="cuda")
    got = edge.norm(x, w, residual=r, bits8=True, out16=True, into={"q": qs[:, shift:shift + dim]})
    check(got, x, w, 1e-6, r, shift)
    assert (qs[:, :shift] == 99).all() and (qs[:, shift + dim:] == 99).all()
    for target in ("x", "residual"):
        x2, r2 = wide.clone()[:, shift:shift + dim], r.clone()
        got2 = edge.norm(x2, w, residual=r2, bits8=True, out16=True, into={"sum": x2 if target == "x" else r2})
        for key in ("sum", "out", "q", "scale"):
            assert torch.equal(got2[key], got[key]), (target, key)


def test_norm_zero_rows_tiny_rows_and_non_finite_values():
    x, _, w = inputs(6, 300, F32, False)
    x[1] = 0
    x[2] *= 1e-25           # far below eps: y is tiny, but no zero row
    x[3, 7] = float("nan")
    x[4, 299] = float("inf")
    x[5, 0] = -float("inf")
    got = edge.norm(x, w, eps=1e-6, bits8=True, out16=True)
    check({k: v[:3] if v is not None else None for k, v in got.items()}, x[:3], w, 1e-6, None, "finite rows")
    assert got["scale"][1] == 0 and (got["q"][1] == 0).all() and (got["out"][1] == 0).all()
    assert got["scale"][3:].isnan().all() and got["out"][3].isnan().all()
    assert got["out"][4, 299].isnan() and (got["out"][4, :299] == 0).all()
    # eps = 0: a row of zeros is 0 / 0
    assert edge.norm(torch.zeros(2, 8, device="cuda"), torch.ones(8, device="cuda"), eps=0.0)["out"].isnan().all()


def test_norm_one_row_between_others_and_on_another_stream():
    x, r, w = inputs(40, 4096, F16, True)
    all_rows = edge.norm(x, w, residual=r, bits8=True)
    one = edge.norm(x[17:18], w, residual=r[17:18], bits8=True)
    assert torch.equal(one["q"][0], all_rows["q"][17]) and torch.equal(one["scale"][0], all_rows["scale"][17])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = edge.norm(x, w, residual=r, bits8=True, stream=side.cuda_stream)
    side.synchronize()
    for key in ("sum", "q", "scale"):
        assert torch.equal(got[key], all_rows[key])
    assert edge.norm(x[:0], w, residual=r[:0], bits8=True)["q"].shape == (0, 4096)


@pytest.mark.parametrize("rows,dim", [(2000, 4096), (3000, 1000), (600, 16384)])
def test_codes_are_the_division_of_the_rows_by_their_scale(rows, dim):
    """binary32 rows come out as they are divided: every code is the nearest integer to out / scale, ties to even."""
    x, r, w = inputs(rows, dim, F32, True, seed=dim)
    got = edge.norm(x, w, residual=r, bits8=True, out16=True)
    want = torch.round(got["out"].cpu() / got["scale"].cpu()[:, None])
    assert torch.equal(got["q"].cpu().float(), want), (got["q"].cpu().float() != want).sum()


@pytest.mark.parametrize("exponent", [-95, -105, -118, -126, -133, -140])
@pytest.mark.parametrize("rows,dim", [(5, 300), (4, 3000), (3, 16384)])
def test_rows_of_the_smallest_values_are_no_rows_of_zeros(rows, dim, exponent):
    """The scale is max / 127 as far as binary32 has it (a subnormal one in the end), codes stay within 127."""
    x, _, w = inputs(rows, dim, F32, False, seed=dim)
    w = torch.full_like(w, 2.0 ** exponent)
    got = {k: v.cpu() for k, v in edge.norm(x, w, bits8=True, out16=True).items() if v is not None}
    top = got["out"].abs().amax(dim=1)
    assert (got["scale"] > 0).all() and torch.equal(got["scale"], top / 127)
    want = torch.round(got["out"] / got["scale"][:, None]).clamp(-127, 127)
    assert torch.equal(got["q"].float(), want) and (got["q"].abs() > 0).any(dim=1).all()


def test_a_scale_that_binary32_does_not_have_is_a_row_of_zeros():
    got = edge.norm(torch.ones(2, 100, device="cuda"), torch.full((100,), 2.0 ** -147, device="cuda"), bits8=True)
    assert (got["scale"] == 0).all() and (got["q"] == 0).all()


@pytest.mark.parametrize("dtype,size,eps", [(BF16, 1e25, 1e-5), (F32, 1e37, 1e-5), (F32, 2e19, 1.0), (BF16, 1e-25, 0.0),
                                            (F32, 1e-36, 0.0), (F32, 3e-20, 1e-38), (F32, 1e-30, 1e-38)])
@pytest.mark.parametrize("rows,dim", [(5, 100), (1500, 1000), (6, 4096), (3, 16384)])
def test_rows_whose_squares_leave_binary32(rows, dim, dtype, size, eps):
    """Rows so large or small that the sum of their squares is no binary32 number, between ordinary ones."""
    x, r, w = inputs(rows, dim, dtype, True, seed=rows + dim)
    x[::2] *= size
    r[::2] *= size
    for residual in (None, r):
        got = edge.norm(x, w, eps=eps, residual=residual, bits8=True, out16=True)
        check(got, x, w, eps, residual, (rows, dim, dtype, size, eps, residual is not None))


@pytest.mark.parametrize("rows,dim,dtype", [((1 << 26) + 5, 8, BF16), ((1 << 24) + 3, 1100, BF16)])
def test_more_rows_than_one_dimension_of_a_grid(rows, dim, dtype):
    w = torch.ones(dim, dtype=dtype, device="cuda")
    x = torch.empty(rows, dim, dtype=dtype, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(0))
    got = edge.norm(x, w, bits8=True, out16=True)
    for part in (slice(0, 1000), slice(rows // 2, rows // 2 + 1000), slice(rows - 1000, rows)):
        check({k: v[part] if v is not None else None for k, v in got.items()}, x[part], w, 1e-6, None, part)
    del x
    assert (got["scale"] > 0).all() and got["q"].view(-1)[::dim].numel() == rows


def test_buffers_for_some_outputs_or_none():
    x, r, w = inputs(30, 500, BF16, True)
    want = edge.norm(x, w, residual=r, bits8=True, out16=True)
    for names in ((), ("sum",), ("q", "out"), ("scale",), ("sum", "out", "q", "scale")):
        into = {k: torch.empty_like(want[k]) for k in names}
        got = edge.norm(x, w, residual=r, bits8=True, out16=True, into=into)
        for key in want:
            assert torch.equal(got[key], want[key]) and (key not in into or got[key] is into[key]), (names, key)
