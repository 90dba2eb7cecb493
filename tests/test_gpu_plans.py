"""Every tile shape, split and tail that the planner chooses for the dense operators' products, at the cheapest
sizes that take it, against float64 under the bounds of the operators' own tests; and that these are all.
"""
import importlib.util
import math
import os
import random

import pytest

torch = pytest.importorskip("torch")
pytest.importorskip("paper_2408_14267_amd.fqt", reason="libfqt.so not built")
from paper_2408_14267_amd import dense as d  # noqa: E402

# kind of a plan: the tile edges of its launches (64, 128, 256; 256 and 64: a tail in small tiles), split or not
FORWARD = {                                 # bf16 operands
    ((64,), False): (65, 129, 127), ((64,), True): (300, 512, 4608),
    ((128,), False): (385, 7451, 79), ((128,), True): (4619, 65, 7187),
    ((256,), False): (2565, 3411, 72), ((256,), True): (3623, 699, 8914), ((256, 64), False): (2818, 5745, 70)}
CODES = {                                   # int8 and e4m3
    ((64,), False): (65, 129, 127), ((64,), True): (64, 1000, 25088),
    ((128,), False): (385, 7451, 79), ((128,), True): (79, 4215, 13287),
    ((256,), False): (2565, 3411, 80), ((256,), True): (548, 6791, 11163), ((256, 64), False): (2818, 5745, 70)}
DX = {((64,), False): (257, 255, 192), ((64,), True): (9, 1784, 76),
      ((128,), False): (89, 13, 24945), ((128,), True): (4705, 7276, 65),
      ((256,), False): (829, 16, 9408), ((256,), True): (132, 6816, 11859), ((256, 64), False): (4157, 10, 4113)}
DW = {((64,), False): (257, 255, 192), ((64,), True): (2052, 11, 93),
      ((128,), False): (6, 133, 16600), ((128,), True): (6260, 4320, 75),
      ((256,), False): (5, 647, 12404), ((256,), True): (7262, 164, 11273), ((256, 64), False): (5, 2483, 7414)}
GRAM = {((64,), False): (67, 66), ((64,), True): (65, 710), ((128,), False): (3102, 3140),
        ((128,), True): (3406, 1457), ((256,), False): (4598, 4501), ((256,), True): (2186, 3448),
        ((256, 64), False): (5726, 5677)}
POLY = {((64,), False): (67, 66), ((128,), False): (3102, 3140), ((128,), True): (2003, 2026),
        ((256,), False): (4598, 4501), ((256,), True): (2912, 2817), ((256, 64), False): (5726, 5677)}
APPLY = {((64,), False): (67, 66), ((128,), False): (74, 24981), ((256,), False): (421, 24625),
         ((256, 64), False): (648, 22959)}


def kind(p):
    return tuple(p.tile[i] for i in range(p.launches)), p.splits > 1


def operators(name):
    spec = importlib.util.spec_from_file_location(name, os.path.join(os.path.dirname(__file__), name + ".py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("cases,product,xt", [(FORWARD, "forward", "bf16"), (CODES, "forward", "int8"),
                                              (CODES, "forward", "e4m3"), (DX, "dx", "bf16"), (DW, "dw", "bf16")])
def test_linear_cases_take_their_plans_and_no_other_is_chosen(cases, product, xt):
    for want, size in cases.items():
        assert kind(d.fqt_linear_plan(d.linear_desc(*size, x_dtype=xt), product)) == want, size
    rng = random.Random(0)
    for _ in range(5000):
        size = [round(math.exp(rng.uniform(math.log(5), math.log(hi)))) for hi in (16384, 8192, 25088)]
        assert kind(d.fqt_linear_plan(d.linear_desc(*size, x_dtype=xt), product)) in cases, size


@pytest.mark.parametrize("cases,product", [(GRAM, "gram"), (POLY, "poly"), (APPLY, "apply")])
def test_ortho_cases_take_their_plans_and_no_other_is_chosen(cases, product):
    for want, size in cases.items():
        assert kind(d.fqt_ortho_plan(d.ortho_desc(*size), product)) == want, size
    rng = random.Random(0)
    for _ in range(5000):
        size = [round(math.exp(rng.uniform(math.log(65), math.log(hi)))) for hi in (16384, 25088)]
        assert kind(d.fqt_ortho_plan(d.ortho_desc(*size), product)) in cases, size


@pytest.mark.gpu
@pytest.mark.parametrize("size", FORWARD.values())
def test_forward(size):
    t = operators("test_gpu_linear")
    t.check_forward(*size, "bf16", "bf16", "gelu", True, True, True)
    t.check_forward(*size, "bf16", "f32", "none", False, False, False)


@pytest.mark.gpu
@pytest.mark.parametrize("size", CODES.values())
@pytest.mark.parametrize("xt", ["int8", "e4m3"])
def test_forward_of_codes(size, xt):
    operators("test_gpu_linear").check_forward(*size, xt, "bf16", "silu", True, True, True)


@pytest.mark.gpu
@pytest.mark.parametrize("size", sorted({*DX.values(), *DW.values()}))
@pytest.mark.parametrize("xt", ["bf16", "e4m3"])
def test_backward(size, xt):
    operators("test_gpu_linear").check_backward(*size, xt, "bf16", "relu")


@pytest.mark.gpu
@pytest.mark.parametrize("size", sorted({*GRAM.values(), *POLY.values(), *APPLY.values()}))
def test_orthogonalisation(size):
    t = operators("test_gpu_ortho")
    rows, cols = size
    g = t.gen(rows, 8, seed=1) @ t.gen(8, cols, seed=2) + 0.3 * t.gen(rows, cols, seed=3)
    raw = torch.full((rows * cols + 64,), 7.0, device="cuda")
    o = raw[:rows * cols].view(rows, cols)
    desc = d.ortho_desc(rows, cols)
    ws = d.ortho_workspace(desc).fill_(0xFF)
    d.fqt_orthogonalize(desc, g, o, ws)
    assert (raw[rows * cols:] == 7).all()
    assert t.off(o, t.ns64(g)) <= t.BOUND["f32"]
    again = torch.empty_like(o)
    d.fqt_orthogonalize(desc, g, again, ws)
    assert torch.equal(again, o)
