"""Codes of rows whose scale is no float32, and the row quantiser over both input types."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TOP = {"int8": 127.0, "e4m3": 448.0}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def dense():
    from paper_2408_14267_amd import dense as d
    return d


def gen(*shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + sum(shape))
    return torch.randn(shape, generator=g, device="cuda")


@pytest.mark.parametrize("cols", [8, 300, 5000, 17000])
@pytest.mark.parametrize("qt", ["int8", "e4m3"])
def test_codes_are_zero_where_the_scale_is(cols, qt):
    """A row of 2^-149 (its maximum over T rounds to 0), and one whose squares have no float32 sum (rstd, y
    and the scale are 0): a code times its scale is 0 for both, and so is the code."""
    d = dense()
    q = torch.empty(2, cols, device="cuda").to(d._TORCH_OF[d.dtype_code(qt)])
    scale, rstd, y = torch.empty(2, device="cuda"), torch.empty(2, device="cuda"), torch.empty(2, cols, device="cuda")
    x = gen(2, cols, seed=1)
    x[0] = 2.0 ** -149
    desc = d.norm_desc(2, cols, x_dtype="f32", q_dtype=qt)
    d.fqt_quantize_rows(desc, x, q, scale)
    assert scale[0] == 0 and (q[0].float() == 0).all()
    assert scale[1] > 0 and q[1].float().abs().amax() == TOP[qt]
    x[0] = 1e25
    d.fqt_rmsnorm_forward(desc, x, torch.ones(cols, device="cuda"), y=y, q=q, scale=scale, rstd=rstd)
    assert rstd[0] == 0 and scale[0] == 0 and (y[0] == 0).all() and (q[0].float() == 0).all()
    assert scale[1] > 0 and q[1].float().abs().amax() == TOP[qt]


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 25088), (5, 7), (300, 513), (1000, 4096), (33, 20001)])
@pytest.mark.parametrize("xt", ["bf16", "f32"])
@pytest.mark.parametrize("qt", ["int8", "e4m3"])
def test_row_quantiser(rows, cols, xt, qt):
    """scale = max |x| / T to a float32 rounding or two; a code is off its quotient by half a step and what
    three float32 products leave of it, 4e-7."""
    d = dense()
    x = (gen(rows, cols, seed=2) * torch.exp(4 * gen(rows, 1, seed=3))).to(DT[xt])
    raw = torch.full((rows * cols + 64,), 5, dtype=torch.uint8, device="cuda")
    q = raw[:rows * cols].view(rows, cols).view(d._TORCH_OF[d.dtype_code(qt)])
    scale = torch.empty(rows, device="cuda")
    d.fqt_quantize_rows(d.norm_desc(rows, cols, x_dtype=xt, q_dtype=qt), x, q, scale)
    assert (raw[rows * cols:] == 5).all()
    s64 = x.double().abs().amax(dim=1) / TOP[qt]
    assert ((scale.double() - s64).abs() <= 3e-7 * s64).all()
    v = x.double() / s64[:, None]
    step = torch.ones_like(v) if qt == "int8" else torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    assert ((q.float().double() - v).abs() <= 0.5 * step + 4e-7 * v.abs()).all()
