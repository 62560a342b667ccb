"""The network operators at the edges of what include/fbdt.h promises of them, against
definitions in 64 bits or the same call in another form."""
import numpy as np
import pytest
import torch

import network_ref as R
import paper_1609_06119_amd as fb
from test_gpu_network import BF16, DEV, F16, F32, SUM_STEPS, check_packed, gen, normal

pytestmark = pytest.mark.gpu


# ---- fast sums -------------------------------------------------------------------

# The 8-bit matrix unit cuts each product, towards zero, off 2^-13 below the largest of its
# group of 8.  That rule carried out in 64 bits on packed normal data leaves errors of
# 2.0e-5 to 2.1e-5 of the result's 2-norm at 64 to 9,000 columns alike; the float32 sums of
# the groups add less than 1e-6.  Held to 3e-5, as 512 results or more vary by a few hundredths.
FAST_NORM = 3e-5


@pytest.mark.parametrize("m,n", [(1, 700), (8, 200), (16, 500), (40, 64), (300, 257), (1025, 1100)])
@pytest.mark.parametrize("k", [64, 129, 640, 2560, 9000])
def test_fast_sums_are_as_near_as_documented(m, n, k):
    a, b = fb.pack(normal(m, m, k)), fb.pack(normal(n, n, k))
    A, B = R.unpack(a)[0], R.unpack(b)[0]
    ref = A @ B.T
    got = R.f64(fb.packed_product(a, b, dtype=F32, fast=True))
    assert np.linalg.norm(got - ref) <= FAST_NORM * np.linalg.norm(ref)


# widths of every remainder by the 4 blocks that a wavefront of the few-rows kernel takes, and
# by the 32 of a workgroup, whole and ending inside a block
@pytest.mark.parametrize("fast", [False, True])
@pytest.mark.parametrize("m", [1, 2, 8, 9, 16])
@pytest.mark.parametrize("k", [1, 17, 100, 128, 129, 250, 256, 300, 384, 400, 512, 513, 640, 1025, 1300,
                               3968, 4096, 4097, 4224, 4480, 4700, 5120, 8192, 8300])
def test_few_rows_are_exact_on_whole_numbers(m, k, fast):
    """Whole numbers of up to 2: no product is 2^-13 of another, sums stay below 2^24."""
    for n in (1, 16, 333):
        a = torch.randint(-2, 3, (m, k), generator=gen(m), device=DEV).float()
        b = torch.randint(-2, 3, (n, k), generator=gen(n + k), device=DEV).float()
        got = fb.packed_product(fb.pack(a), fb.pack(b), dtype=F32, fast=fast)
        assert torch.equal(got, a @ b.t())


# ---- the weights' gradient of one row -----------------------------------------------

@pytest.mark.parametrize("n", [1, 5, 8, 40, 333])
@pytest.mark.parametrize("stride", [None, 2 ** 22 + 8, 2 ** 26, 2 ** 31, 2 ** 31 + 8, 2 ** 40 + 24])
def test_weight_grad_of_one_row_at_any_stride(n, stride):
    """A single row's stride means nothing: the rows that a step has beside it are no rows,
    and add nothing to values that are infinite.  NaN lies where they would begin."""
    from paper_1609_06119_amd._lib import check, lib
    k = 200
    wide = torch.full((70 * 340,), float("nan"), dtype=BF16, device=DEV)
    dy = wide[:n]
    dy.copy_(normal(n, n, dtype=BF16))
    dy[n // 2] = float("inf")
    x = fb.pack(1 + normal(2, 1, k).abs())             # (no zeros: inf * 0 is NaN)
    out = torch.empty((n, k), device=DEV)
    L = lib()
    args = (dy.data_ptr(), n if stride is None else stride, 1, n)
    assert L.fbdt_packed_weight_grad_work(*args, k) == 0
    check("fbdt_packed_weight_grad", L.fbdt_packed_weight_grad(
        *args, x.data.data_ptr(), x.data.shape[1], x.scales.data_ptr(), x.scales.shape[1], k,
        out.data_ptr(), 0, k, None, 0, torch.cuda.current_stream().cuda_stream))
    want = R.f64(dy)[:, None] * R.unpack(x)[0]         # 8 + 4 significant bits: exact
    assert np.array_equal(R.f64(out), want)


# ---- gradients that torch would record ------------------------------------------------

def test_tensors_whose_gradient_is_recorded_are_refused():
    """The calls build no graph: a gradient that torch waits for would be dropped."""
    x, gain = normal(1, 4, 200), torch.ones(200, device=DEV)
    t = torch.zeros(4, dtype=torch.int32, device=DEV)
    p = fb.pack(x)
    rstd = torch.ones(4, device=DEV)
    asked, asked_gain, asked_16 = (v.clone().requires_grad_() for v in (x, gain, x.bfloat16()))
    calls = {
        "embed": lambda: fb.embed(asked, t), "out": lambda: fb.embed(x, t, out=asked * 1),
        "embed_grad": lambda: fb.embed_grad(t, asked, 5),
        "embed_grad of nothing": lambda: fb.embed_grad(t[:0], asked[:0], 5),
        "rms_norm": lambda: fb.rms_norm(asked, gain), "gain": lambda: fb.rms_norm(x, asked_gain),
        "residual": lambda: fb.rms_norm(x, gain, residual=asked),
        "rms_norm_grad": lambda: fb.rms_norm_grad(asked, x, gain, rstd),
        "dh": lambda: fb.rms_norm_grad(x, x, gain, rstd, dh=asked), "pack": lambda: fb.pack(asked),
        "product": lambda: fb.packed_product(p, p, dtype=F32, out=asked[:, :4] * 1),
        "weight_grad": lambda: fb.packed_weight_grad(asked_16, p),
    }
    for name, call in calls.items():
        with pytest.raises(ValueError, match="requires grad"):
            call()
            pytest.fail(name)
        with torch.no_grad():
            if name not in ("out", "product"):
                call()
        with torch.inference_mode():
            call()
    with torch.no_grad():
        assert torch.equal(fb.rms_norm(asked, asked_gain).y, fb.rms_norm(x, gain).y)


# ---- results beside and on what a call reads --------------------------------------------

def test_results_on_inputs_are_refused_and_beside_them_are_not():
    wide = normal(1, 60, 100)
    table = wide[:, :40]
    t = torch.randint(0, 60, (60,), generator=gen(2), device=DEV)
    want = table[t]
    fb.embed(table, t, out=wide[:, 50:90])                     # columns of one matrix
    assert torch.equal(wide[:, 50:90], want)
    d = normal(3, 60, 40)
    a, x = fb.pack(normal(4, 60, 200)), normal(5, 60, 40, dtype=BF16)
    g = fb.embed_grad(t, d, 60)
    fb.embed_grad(t, d, 60, out=wide[:, 50:90])
    assert torch.equal(wide[:, 50:90], g)
    codes = fb.Codes(torch.zeros((3, 64), dtype=torch.uint8, device=DEV), 10)
    for call in (lambda: fb.embed(table, t[:30], out=table[:30]), lambda: fb.embed_grad(t, d, 60, out=d),
                 lambda: fb.event_tokens(codes, 16, out=codes.data.view(torch.int32).view(-1)[:30].view(10, 3)),
                 lambda: fb.packed_product(a, a, dtype=F32, out=a.data.view(F32)[:, :60]),
                 lambda: fb.packed_weight_grad(x, a, dtype=BF16, out=torch.as_strided(x, (40, 200), (1, 1)))):
        with pytest.raises((fb.FbdtError, ValueError), match="overlap"):
            call()


# ---- the norm in place --------------------------------------------------------------------

def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("dtype,code", [(F32, 0), (BF16, 1)])
@pytest.mark.parametrize("n,width", [(70, 24), (9, 500), (70, 2560), (5, 9000), (5, 28_001), (600, 33_000)])
@pytest.mark.parametrize("packed", [False, True])
def test_h_takes_the_place_of_x_or_the_residual(n, width, dtype, code, packed):
    from paper_1609_06119_amd._lib import check, lib
    x, r, gain = normal(1, n, width, dtype=dtype), normal(2, n, width, dtype=dtype), normal(3, width)
    want = fb.rms_norm(x, gain, residual=r, packed=packed)
    for place in ("x", "residual"):
        a, b, rstd = x.clone(), r.clone(), torch.empty(n, device=DEV)
        h = a if place == "x" else b
        if packed:
            y = fb.Packed.empty(n, width)
            to = (None, 0, y.data.data_ptr(), y.data.shape[1], y.scales.data_ptr(), y.scales.shape[1])
        else:
            y = torch.empty_like(x)
            to = (y.data_ptr(), width, None, 0, None, 0)
        check("fbdt_rms_norm", lib().fbdt_rms_norm(
            a.data_ptr(), width, b.data_ptr(), width, code, n, width, gain.data_ptr(), 1e-6, h.data_ptr(),
            width, *to, rstd.data_ptr(), stream()))
        assert torch.equal(h, want.h) and torch.equal(rstd, want.rstd)
        assert torch.equal(b if place == "x" else a, r if place == "x" else x)
        assert torch.equal(y.unpack(), want.y.unpack()) if packed else torch.equal(y, want.y)


@pytest.mark.parametrize("dtype,code", [(F32, 0), (BF16, 1)])
@pytest.mark.parametrize("n,width", [(70, 24), (9, 500), (70, 2560), (70, 4000), (5, 9000), (600, 17_001)])
def test_dx_takes_the_place_of_dy_or_dh(n, width, dtype, code):
    from paper_1609_06119_amd._lib import check, lib
    dy, h, dh = (normal(s, n, width, dtype=dtype) for s in (1, 2, 3))
    gain, rstd = normal(4, width), 0.5 + normal(5, n).abs()
    want, want_gain = fb.rms_norm_grad(dy, h, gain, rstd, dh=dh)
    L = lib()
    need = L.fbdt_rms_norm_grad_work(n, width)
    work = torch.empty(need, dtype=torch.uint8, device=DEV)
    for place in ("dy", "dh"):
        a, b, dgain = dy.clone(), dh.clone(), torch.empty(width, device=DEV)
        dx = a if place == "dy" else b
        check("fbdt_rms_norm_grad", L.fbdt_rms_norm_grad(
            a.data_ptr(), width, h.data_ptr(), width, b.data_ptr(), width, code, n, width, gain.data_ptr(),
            rstd.data_ptr(), dx.data_ptr(), width, dgain.data_ptr(), work.data_ptr(), need, stream()))
        assert torch.equal(dx, want) and torch.equal(dgain, want_gain)
        assert torch.equal(b if place == "dy" else a, dh if place == "dy" else dy)


# ---- 8-bit rows ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("width", [4100, 9504, 14_000, 20_000, 24_577, 25_000, 28_672, 32_640, 32_768, 32_769])
def test_wide_rows_packed(dtype, width):
    """The codes of rows by 256 lanes to 1024 and of those that are read twice."""
    x, gain = normal(1, 7, width, dtype=dtype, scale=2.0), 1 + normal(3, width, scale=0.2)
    x[2] = 0.0
    p = fb.rms_norm(x, gain, eps=1e-4, packed=True)
    ry, _, _ = R.rms_norm(R.f64(x), None, R.f64(gain), np.float64(np.float32(1e-4)))
    check_packed(p.y, ry, (SUM_STEPS + 16) * R.U32)
    assert not R.f64(p.y.data)[:, width:].any()


@pytest.mark.parametrize("m,n,k", [(3, 2, 1), (3, 9, 200), (200, 40, 384), (4100, 300, 130)])
def test_a_scale_that_is_nan(m, n, k):
    """It makes its block NaN whatever its codes are, 0 among them, and nothing else."""
    x, w = fb.pack(1 + normal(1, m, k).abs()), fb.pack(1 + normal(2, n, k).abs())
    row, block = m // 2, (k - 1) // 128
    x.scales.view(torch.uint8)[row, block] = 255
    x.data.view(torch.uint8)[row, 128 * block] = 0
    nan = np.zeros((m, n), dtype=bool)
    nan[row] = True
    for fast in (False, True):
        assert np.array_equal(np.isnan(R.f64(fb.packed_product(x, w, dtype=F32, fast=fast))), nan)
        assert np.array_equal(np.isnan(R.f64(fb.packed_product(w, x, dtype=F32, fast=fast))), nan.T)
    dy = 1 + normal(3, m, n, dtype=BF16).abs()
    got = R.f64(fb.packed_weight_grad(dy, x))
    nan = np.zeros((n, k), dtype=bool)
    nan[:, 128 * block:] = True
    assert np.array_equal(np.isnan(got), nan)
    keep = ~nan[0]
    Y, X = R.f64(dy), R.unpack(x)[0][:, keep]
    assert (np.abs(got[:, keep] - Y.T @ X) <= (m + 3) * R.U32 * (Y.T @ X)).all()


def test_packed_rows_of_one_row():
    """A row of packed rows is what it is among the others, whatever its tensors hold beside it."""
    a, b, x = fb.pack(normal(1, 3, 300)), fb.pack(normal(2, 40, 300)), normal(3, 3, 60, dtype=BF16)
    want = fb.packed_product(a, b, dtype=F32)
    for held in (384, 300 + 128):
        for blocks in (3, 4):
            data = torch.zeros((3, 512), dtype=torch.uint8, device=DEV)
            data[:, :384] = a.data.view(torch.uint8)
            scales = torch.zeros((3, 8), dtype=torch.uint8, device=DEV)
            scales[:, :4] = a.scales.view(torch.uint8)
            data, scales = data.view(a.data.dtype), scales.view(a.scales.dtype)
            for rows in (slice(0, 3), slice(1, 2)):
                p = fb.Packed(data[rows, :held], scales[rows, :blocks], 300)
                assert torch.equal(fb.packed_product(p, b, dtype=F32), want[rows])
                got = fb.packed_weight_grad(x[rows], p)
                assert torch.equal(got, fb.packed_weight_grad(x[rows], fb.pack(p.unpack())))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(1, 10_240, 2560), (1, 40, 9000), (5, 1280, 1280), (8, 777, 1300),
                                   (16, 500, 640)])
def test_few_rows_are_added_in_full(m, n, k, dtype):
    """The 8-bit unit's sums would save them next to nothing: fast gives the same bits."""
    a, b = fb.pack(normal(m, m, k)), fb.pack(normal(n, n, k))
    want = fb.packed_product(a, b, dtype=dtype)
    assert torch.equal(fb.packed_product(a, b, dtype=dtype, fast=True), want)
