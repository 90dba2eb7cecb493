"""Softmax cross entropy of a linear layer, and its gradients, against the formulas in float64.

Tolerances, with u = 2^-24.  On operands whose sums float32 holds exactly (small integers times powers of two),
z is exact; y = z log2(e) is off by u |y| / 2 and the constant's u / 3 of |y - top|, so an exponential, with |z| <= 40 and |z -
top| <= 40 here, by 2 * 29 u + 20 u + 29 u, its difference's rounding, and its instruction's 2 u: 140 u; at most 80 additions one
after the other join them, each with an exponential of a difference: their sum is off by 200 u + 80 * 4 u = 520 u at most, and
with it log1p of it, lse and loss, relative to log1p of the sum; lse, loss and smoothing add their own roundings of 8 u of the
terms.
Other operands: z is off by (K + 8) u of the sum of |x w| and the bias, which enters lse once and loss twice.
Gradients: dz in float32 by 600 u and z's error relative to its terms, then 2^-8 for bf16, carried to dx and dw with the
magnitudes of the terms; sums of n terms n u of the sum of magnitudes; outputs in bf16 2^-8.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
IGNORE = -100


def step():
    from paper_2408_14267_amd import step as s
    return s


def make(M, N, K, kind, seed=0, integers=False, bias=True, ignored=0.2, ldx=0, ldw=0):
    """Operands as a dict, with their float64 values x64, w64."""
    g = torch.Generator(device="cuda").manual_seed(seed * 104729 + 31 * M + 7 * N + K)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def strided(t, ld):
        if not ld:
            return t
        raw = torch.full((t.shape[0] * ld + 64,), 3, device="cuda").to(t.dtype)
        v = raw[:t.shape[0] * ld].view(t.shape[0], ld)[:, :t.shape[1]]
        v.copy_(t)
        return v

    o = {}
    if integers:
        # z = integers / 8, |z| about 2 sqrt(K) / 8 wide: held by few non-zeros in x
        x = torch.randint(-2, 3, (M, K), generator=g, device="cuda").float()
        x *= torch.rand(M, K, generator=g, device="cuda") < min(1.0, 200.0 / max(K, 1))
        w = torch.randint(-2, 3, (N, K), generator=g, device="cuda").float()
        if kind == "bf16":
            w /= 8
        sx, sw = torch.full((M,), 0.5, device="cuda"), torch.full((N,), 0.25, device="cuda")
        b = torch.randint(-8, 9, (N,), generator=g, device="cuda").float() / 8
    else:
        x, w = 1.5 * normal(M, K), normal(N, K) / math.sqrt(max(K, 1))
        sx = sw = None
        b = normal(N)
    if kind == "bf16":
        o["x"], o["w"] = x.bfloat16(), w.bfloat16()
        o["x_scale"] = o["w_scale"] = None
    else:
        top, dt = (127.0, torch.int8) if kind == "int8" else (448.0, torch.float8_e4m3fn)
        if sx is None:
            sx = x.abs().amax(dim=1).clamp_min(1e-20) / top if K else torch.ones(M, device="cuda")
            sw = w.abs().amax(dim=1).clamp_min(1e-20) / top if K else torch.ones(N, device="cuda")
            x, w = x / sx[:, None], w / sw[:, None]
            if kind == "int8":
                x, w = x.round(), w.round()
        o["x"], o["w"], o["x_scale"], o["w_scale"] = x.to(dt), w.to(dt), sx, sw
    o["x64"], o["w64"] = o["x"].float().double(), o["w"].float().double()
    if o["x_scale"] is not None:
        o["x64"], o["w64"] = o["x64"] * sx.double()[:, None], o["w64"] * sw.double()[:, None]
    o["x"], o["w"] = strided(o["x"], ldx), strided(o["w"], ldw)
    o["bias"] = b if bias else None
    t = torch.randint(0, N, (M,), generator=g, device="cuda")
    out = torch.rand(M, generator=g, device="cuda") < ignored
    o["target"] = torch.where(out, IGNORE, t)
    return o


def reference(o, smoothing=0.0):
    """z, lse, loss, which rows count, the error of z."""
    z = o["x64"] @ o["w64"].t().contiguous()
    mag = o["x64"].abs() @ o["w64"].abs().t().contiguous()
    if o["bias"] is not None:
        z, mag = z + o["bias"].double(), mag + o["bias"].double().abs()
    lse = torch.logsumexp(z, dim=1)
    counted = o["target"] != IGNORE
    t = o["target"].clamp(min=0)
    rest = torch.exp(z - z.amax(dim=1, keepdim=True))
    rest.scatter_(1, z.argmax(dim=1, keepdim=True), 0.0)
    tail = torch.log1p(rest.sum(dim=1))                     # lse - top, exactly enough when it is tiny
    top = z.amax(dim=1)
    loss = (1 - smoothing) * (top - z.gather(1, t[:, None])[:, 0]) + tail
    if smoothing:
        loss = loss + smoothing * (top - z.mean(dim=1))
    zerr = ((o["x"].shape[1] + 8) * U * mag).amax(dim=1)
    return z, lse, torch.where(counted, loss, 0.0), counted, zerr, tail


def forward(o, M, N, K, kind, smoothing=0.0, mean=True, **kw):
    s = step()
    desc = s.loss_desc(M, N, K, x_dtype=kind, smoothing=smoothing, ignore=IGNORE, **kw)
    loss, lse = torch.full((M + 3,), 7.0, device="cuda"), torch.full((M + 3,), 7.0, device="cuda")
    out = torch.full((4,), 7.0, device="cuda")
    ws = s.loss_workspace(desc)
    s.fqt_loss_forward(desc, o["x"], o["w"], o["target"], loss[:M], lse[:M], ws, bias=o["bias"], x_scale=o["x_scale"],
                       w_scale=o["w_scale"], mean=out[:2] if mean else None)
    assert (loss[M:] == 7).all() and (lse[M:] == 7).all() and (out[2:] == 7).all()
    return loss[:M], lse[:M], out[:2]


def check_forward(o, M, N, K, kind, smoothing=0.0, exact_sums=False, **kw):
    loss, lse, mean = forward(o, M, N, K, kind, smoothing, **kw)
    z, lse64, loss64, counted, zerr, tail = reference(o, smoothing)
    if exact_sums:
        zerr = torch.zeros_like(zerr)
    big = z.abs().amax(dim=1)
    lim = 520 * U * tail + 8 * U * big + zerr
    err = (lse.double() - lse64).abs()
    assert (err <= lim).all(), f"lse off by {(err / lim).max().item():.3g} of the bound"
    # smoothing: a mean of N terms, off by (N + 8) u of the largest
    lim = 520 * U * tail + 8 * U * loss64.abs() + 2 * zerr + (smoothing * 2 * (N + 8) * U * big if smoothing else 0.0)
    err = (loss.double() - loss64).abs()
    assert (loss[~counted] == 0).all()
    assert (err <= lim + 1e-300).all(), f"loss off by {(err / lim.clamp_min(1e-300)).max().item():.3g} of the bound"
    n = int(counted.sum())
    want = loss.double()[counted].sum() / n if n else torch.zeros((), dtype=torch.float64)
    assert abs(mean[0].item() - want.item()) <= 4 * U * abs(want.item()) + 1e-300
    assert mean[1].item() == pytest.approx(1 / n if n else 0.0, rel=2 * U)


SHAPES = [(1, 1, 8), (1, 10, 64), (1, 4099, 513), (2, 1000, 4096), (4, 65, 1), (3, 32768, 96), (5, 1, 16),
          (5, 7, 3), (16, 1000, 2048), (63, 64, 64), (64, 65, 65), (64, 1000, 4096), (65, 129, 300), (128, 128, 512),
          (129, 255, 72), (130, 10007, 40), (257, 300, 1153), (300, 4096, 256), (513, 2049, 128), (777, 1000, 513),
          (1000, 513, 64), (2049, 130, 64), (2304, 4864, 64), (40, 131072, 16), (5000, 10, 32), (4608, 4097, 72),
          (1100, 9000, 520)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
def test_forward(M, N, K, kind):
    check_forward(make(M, N, K, kind, seed=1), M, N, K, kind)


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_forward_on_exact_sums(M, N, K, kind):
    o = make(M, N, K, kind, seed=2, integers=True, bias=(M + N) % 2 == 0)
    z = reference(o)[0]
    assert (z * 64 == (z * 64).round()).all() and (z.amax(dim=1, keepdim=True) - z).max() < 110
    check_forward(o, M, N, K, kind, exact_sums=True)


@pytest.mark.parametrize("M,N,K,ldx,ldw", [(70, 200, 96, 104, 136), (70, 200, 96, 97, 99), (3, 200, 96, 101, 97),
                                           (300, 600, 64, 64, 80), (300, 600, 64, 72, 64), (20, 1000, 4096, 4099, 4104)])
@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
def test_forward_of_strided_rows(M, N, K, ldx, ldw, kind):
    check_forward(make(M, N, K, kind, seed=3, ldx=ldx, ldw=ldw), M, N, K, kind, ldx=ldx, ldw=ldw)


@pytest.mark.parametrize("M,N,K", [(1, 10, 64), (5, 1000, 256), (64, 1000, 4096), (300, 700, 128), (1500, 4100, 64)])
@pytest.mark.parametrize("smoothing", [0.1, 1.0])
def test_smoothing(M, N, K, smoothing):
    check_forward(make(M, N, K, "e4m3", seed=4), M, N, K, "e4m3", smoothing)
    check_forward(make(M, N, K, "bf16", seed=4), M, N, K, "bf16", smoothing)
    check_forward(make(M, N, K, "int8", seed=4, bias=False), M, N, K, "int8", smoothing)


@pytest.mark.parametrize("M", [1, 3, 20, 400])
def test_small_losses_keep_their_precision(M):
    """The target far above all others: the loss is the sum of their exponentials, relative to itself."""
    N, K = 300, 64
    w = torch.zeros(N, K, device="cuda")
    w[torch.arange(N), torch.arange(N) % 32] = 1.0
    x = torch.zeros(M, K, device="cuda")
    bias = torch.zeros(N, device="cuda")
    bias[7] = 25.0
    o = dict(x=x.bfloat16(), w=w.bfloat16(), x64=x.double(), w64=w.double(), bias=bias, x_scale=None, w_scale=None,
             target=torch.full((M,), 7, device="cuda"))
    loss, lse, _ = forward(o, M, N, K, "bf16")
    want = math.log1p((N - 1) * math.exp(-25.0))
    assert ((loss.double() - want).abs() <= 600 * U * want).all()


@pytest.mark.parametrize("M,N,K", [(2, 300, 64), (30, 1000, 4096), (300, 700, 128)])
def test_classes_that_are_out(M, N, K):
    """A bias of minus infinity takes classes out, whole slots of them too, and all but one."""
    o = make(M, N, K, "bf16", seed=5, ignored=0.0)
    o["bias"][64:256] = -math.inf
    o["target"] = o["target"] % 64
    z, lse64, loss64, _, zerr, tail = reference(dict(o, bias=o["bias"]))
    loss, lse, _ = forward(o, M, N, K, "bf16")
    mag = o["x64"].abs() @ o["w64"].abs().t().contiguous()
    zerr = ((K + 8) * U * (mag + 8)).amax(dim=1)
    lim = 520 * U * tail + 100 * U + 2 * zerr
    assert ((lse.double() - lse64).abs() <= lim).all() and ((loss.double() - loss64).abs() <= lim).all()
    o["bias"][:] = -math.inf
    o["bias"][5] = 0.25
    o["target"][:] = 5
    loss, lse, _ = forward(o, M, N, K, "bf16")
    assert (loss == 0).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("M,N,K", [(3, 100, 64), (40, 100, 4096), (300, 700, 128)])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_targets_that_are_no_class(M, N, K, kind):
    o = make(M, N, K, kind, seed=6, ignored=0.0)
    good = forward(o, M, N, K, kind)[0].clone()
    for bad in (-1, N, N + 1, 1 << 40, -(1 << 62), (1 << 32) + 3):
        t = o["target"].clone()
        t[M // 2] = bad
        loss, _, mean = forward(dict(o, target=t), M, N, K, kind)
        assert torch.isnan(loss[M // 2]) and torch.isnan(mean[0])
        keep = torch.arange(M, device="cuda") != M // 2
        assert torch.equal(loss[keep], good[keep])


def test_no_row_counts():
    for M in (0, 1, 40, 300):
        o = make(M, 50, 64, "bf16", ignored=2.0)
        loss, _, mean = forward(o, M, 50, 64, "bf16")
        assert (loss == 0).all() and (mean == 0).all()


@pytest.mark.parametrize("M,N,K", [(2, 50, 64), (40, 300, 2048), (300, 700, 128)])
def test_nan_stays_in_its_row(M, N, K):
    o = make(M, N, K, "bf16", seed=7, ignored=0.0)
    good = forward(o, M, N, K, "bf16")
    for v in (math.nan, math.inf):
        x = o["x"].clone()
        x[1, 3] = v
        loss, lse, _ = forward(dict(o, x=x), M, N, K, "bf16")
        assert not torch.isfinite(loss[1]) and not torch.isfinite(lse[1])
        keep = torch.arange(M, device="cuda") != 1
        assert torch.equal(loss[keep], good[0][keep]) and torch.equal(lse[keep], good[1][keep])


# ----------------------------------------------------------------------------- gradients

def backward(o, M, N, K, kind, lse, dloss=None, dmean=None, mean=None, smoothing=0.0, dx_dtype="bf16", dw_dtype="bf16",
             lddx=0, lddw=0, want=("dx", "dw", "dbias"), **kw):
    s = step()
    desc = s.loss_desc(M, N, K, x_dtype=kind, dx_dtype=dx_dtype, dw_dtype=dw_dtype, smoothing=smoothing, ignore=IGNORE,
                       lddx=lddx, lddw=lddw, **kw)

    def room(rows, ld, cols, dt):
        ld = ld or cols
        raw = torch.full((rows * ld + 64,), 7, device="cuda").to(DT[dt])
        keep = torch.ones_like(raw, dtype=torch.bool)
        if rows and cols:
            keep[:rows * ld].view(rows, ld)[:, :cols] = False
        return raw[:rows * ld].view(rows, ld)[:, :cols], raw, keep

    rooms = {"dx": room(M, lddx, K, dx_dtype), "dw": room(N, lddw, K, dw_dtype), "dbias": room(1, 0, N, "f32")}
    out = {k: rooms[k][0] for k in want}
    if "dbias" in out:
        out["dbias"] = out["dbias"][0]
    ws = s.loss_workspace(desc, backward=True)
    s.fqt_loss_backward(desc, o["x"], o["w"], o["target"], lse, ws, dloss=dloss, dmean=dmean, mean=mean, bias=o["bias"],
                        x_scale=o["x_scale"], w_scale=o["w_scale"], **out)
    for k in want:
        assert (rooms[k][1][rooms[k][2]].float() == 7).all(), k
    return out


def check_backward(o, M, N, K, kind, smoothing=0.0, reduction="none", dx_dtype="bf16", dw_dtype="bf16", **kw):
    g = torch.Generator(device="cuda").manual_seed(M + N)
    z, lse64, _, counted, zerr, _ = reference(o, smoothing)
    lse = lse64.float()
    if reduction == "none":
        dloss = torch.randn(M, generator=g, device="cuda")
        c = dloss.double()
        got = backward(o, M, N, K, kind, lse, dloss=dloss, smoothing=smoothing, dx_dtype=dx_dtype, dw_dtype=dw_dtype, **kw)
    else:
        n = max(1, int(counted.sum()))
        dmean, mean = torch.tensor([0.75], device="cuda"), torch.tensor([3.0, 1.0 / n], device="cuda")
        c = (dmean.double() * mean.double()[1]).expand(M)
        got = backward(o, M, N, K, kind, lse, dmean=dmean, mean=mean, smoothing=smoothing, dx_dtype=dx_dtype,
                       dw_dtype=dw_dtype, **kw)
    c = torch.where(counted, c, 0.0)
    p = torch.exp(z - lse.double()[:, None])
    q = torch.full_like(z, smoothing / N)
    q.scatter_add_(1, o["target"].clamp(min=0)[:, None], torch.full_like(z[:, :1], 1 - smoothing))
    dz = (p - q) * c[:, None]
    # what dz may be off by in float32, and with its rounding to bf16
    d32 = (p * (600 * U + 2 * zerr[:, None] + 4 * U * lse.double().abs()[:, None]) + 4 * U * (p + q)) * c.abs()[:, None]
    d16 = d32 + HALF * (dz.abs() + d32)
    x, w = o["x64"], o["w64"]
    cases = {"dx": (dz @ w, d16 @ w.abs() + N * U * (dz.abs() @ w.abs()), HALF if dx_dtype == "bf16" else U),
             "dw": (dz.t().contiguous() @ x, d16.t().contiguous() @ x.abs() + M * U * (dz.abs().t().contiguous() @ x.abs()),
                    HALF if dw_dtype == "bf16" else U),
             "dbias": (dz.sum(dim=0), d32.sum(dim=0) + M * U * dz.abs().sum(dim=0), U)}
    for k, t in got.items():
        want, lim, half = cases[k]
        err = (t.double() - want).abs()
        lim = lim + half * (want.abs() + lim) + 1e-37
        assert torch.isfinite(t).all() and (err <= lim).all(), f"{k}: off by {(err / lim).max().item():.3g} of the bound"
    return got


BACK = [(1, 10, 64), (1, 4099, 513), (4, 65, 1), (5, 1, 16), (5, 7, 3), (16, 1000, 2048), (64, 1000, 4096), (65, 129, 300),
        (129, 255, 72), (130, 10007, 40), (257, 300, 1153), (777, 1000, 513), (1000, 513, 64), (2304, 4864, 64),
        (5000, 10, 32), (4608, 4097, 72), (1100, 9000, 520), (512, 8192, 1024), (3000, 257, 2048), (9000, 100, 512)]


@pytest.mark.parametrize("M,N,K", BACK)
@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
def test_backward(M, N, K, kind):
    check_backward(make(M, N, K, kind, seed=8), M, N, K, kind)


@pytest.mark.parametrize("M,N,K", [(5, 7, 3), (64, 1000, 4096), (300, 700, 128)])
@pytest.mark.parametrize("dx_dtype,dw_dtype", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32")])
def test_backward_types(M, N, K, dx_dtype, dw_dtype):
    check_backward(make(M, N, K, "bf16", seed=9, bias=False), M, N, K, "bf16", dx_dtype=dx_dtype, dw_dtype=dw_dtype)


@pytest.mark.parametrize("M,N,K", [(6, 10, 64), (64, 1000, 512), (300, 700, 128)])
@pytest.mark.parametrize("smoothing", [0.0, 0.1, 1.0])
def test_backward_of_the_mean(M, N, K, smoothing):
    check_backward(make(M, N, K, "bf16", seed=10), M, N, K, "bf16", smoothing, reduction="mean")


@pytest.mark.parametrize("want", [("dx",), ("dw",), ("dbias",), ("dx", "dbias"), ("dw", "dbias")])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_backward_of_some(want, kind):
    o = make(200, 300, 96, kind, seed=11)
    both, some = check_backward(o, 200, 300, 96, kind), check_backward(o, 200, 300, 96, kind, want=want)
    for k in want:
        assert torch.equal(both[k], some[k]), k


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_backward_of_strided_rows(kind):
    for ldx, ldw, lddx, lddw in ((97, 99, 101, 103), (104, 96, 96, 120), (96, 104, 100, 96)):
        o = make(150, 260, 96, kind, seed=12, ldx=ldx, ldw=ldw)
        check_backward(o, 150, 260, 96, kind, ldx=ldx, ldw=ldw, lddx=lddx, lddw=lddw)


@pytest.mark.parametrize("M,N,K", [(9000, 20011, 24), (9000, 20480, 64)])
@pytest.mark.parametrize("kind,dx_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("e4m3", "bf16")])
def test_backward_in_pieces(M, N, K, kind, dx_dtype):
    """Sizes whose dz goes through the workspace in several pieces, the last one shorter."""
    s = step()
    desc = s.loss_desc(M, N, K, x_dtype=kind)
    assert s.fqt_loss_workspace_size(desc, True) < M * N * (4 if kind == "e4m3" else 2)
    check_backward(make(M, N, K, kind, seed=13), M, N, K, kind, dx_dtype=dx_dtype)


@pytest.mark.parametrize("kind,M,N,K", [("bf16", 4608, 12288, 1024), ("int8", 4608, 12288, 1024), ("e4m3", 4608, 12288, 1024),
                                        ("bf16", 4608, 16500, 4096)])
def test_large(kind, M, N, K):
    """Sizes that take 256 x 256 tiles, the last in every product, smoothed labels."""
    o = make(M, N, K, kind, seed=24)
    check_forward(o, M, N, K, kind, 0.1)
    check_backward(o, M, N, K, kind, 0.1)


def test_backward_of_rows_that_do_not_count():
    M, N, K = 300, 700, 128
    o = make(M, N, K, "bf16", seed=14, ignored=2.0)
    got = check_backward(o, M, N, K, "bf16")
    assert all((t == 0).all() for t in got.values())
    # whatever z and lse are there
    lse = torch.full((M,), math.nan, device="cuda")
    got = backward(o, M, N, K, "bf16", lse, dloss=torch.ones(M, device="cuda"))
    assert all((t == 0).all() for t in got.values())
    o["target"][:] = 5
    lse = reference(o)[1].float()
    o["target"][17] = N
    got = backward(o, M, N, K, "bf16", lse, dloss=torch.ones(M, device="cuda"))
    assert torch.isnan(got["dx"][17].float()).all() and torch.isfinite(got["dx"][:17].float()).all()


def test_backward_of_no_rows():
    s = step()
    desc = s.loss_desc(0, 40, 16)
    x, w = torch.empty(0, 16, device="cuda").bfloat16(), torch.ones(40, 16, device="cuda").bfloat16()
    dw, dbias = torch.ones(40, 16, device="cuda").bfloat16(), torch.ones(40, device="cuda")
    e = torch.empty(0, device="cuda")
    s.fqt_loss_backward(desc, x, w, torch.empty(0, dtype=torch.int64, device="cuda"), e, s.loss_workspace(desc, True),
                        dloss=e, dw=dw, dbias=dbias)
    assert (dw == 0).all() and (dbias == 0).all()


@pytest.mark.parametrize("M,N", [(1, 1), (3, 10), (300, 700)])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_no_features(M, N, kind):
    """A contraction over nothing: z is the bias."""
    o = make(M, N, 0, kind, seed=22, ignored=0.0)
    check_forward(o, M, N, 0, kind)
    got = check_backward(o, M, N, 0, kind)
    assert got["dx"].shape == (M, 0) and got["dw"].shape == (N, 0)


@pytest.mark.parametrize("M,N,K", [(3, 100, 64), (200, 300, 96)])
def test_ignored_class_numbers(M, N, K):
    """`ignore` may be a class (a padding token): its rows are left out, the class stays in the sums."""
    s = step()
    o = make(M, N, K, "bf16", seed=23, ignored=0.0)
    o["target"][::2] = 7
    desc = s.loss_desc(M, N, K, ignore=7)
    loss, lse, mean = (torch.empty(n, device="cuda") for n in (M, M, 2))
    s.fqt_loss_forward(desc, o["x"], o["w"], o["target"], loss, lse, s.loss_workspace(desc), bias=o["bias"], mean=mean)
    z, lse64, _, _, zerr, _ = reference(o)
    assert (loss[::2] == 0).all() and ((lse.double() - lse64).abs() <= 600 * U * lse64.abs() + zerr).all()
    dx, db = torch.empty_like(o["x"]), torch.empty(N, device="cuda")
    s.fqt_loss_backward(desc, o["x"], o["w"], o["target"], lse, s.loss_workspace(desc, True), dmean=torch.ones(1, device="cuda"),
                        mean=mean, bias=o["bias"], dx=dx, dbias=db)
    assert (dx[::2] == 0).all() and (o["target"] == 7).sum() + round(1 / mean[1].item()) == M
    counted = o["target"] != 7
    want = (torch.exp(z - lse.double()[:, None])[counted].sum(dim=0) - torch.bincount(o["target"][counted], minlength=N)) * mean[1].double()
    assert ((db.double() - want).abs() <= (700 * U + 4 * zerr.max()) * 2 * mean[1].double() * M + 1e-12).all()


def test_gradient_against_differences():
    """The slope of the float64 loss along a direction of x, w and bias, from the gradients and from a difference."""
    M, N, K = 60, 90, 40
    o = make(M, N, K, "bf16", seed=15)
    g = torch.Generator(device="cuda").manual_seed(1)
    dx, dw, db = (torch.randn(*s, generator=g, device="cuda", dtype=torch.float64) for s in ((M, K), (N, K), (N,)))

    def total(h):
        moved = dict(o, x64=o["x64"] + h * dx, w64=o["w64"] + h * dw, bias=o["bias"].double() + h * db)
        return reference(moved, 0.1)[2].sum()

    h = 1e-4
    slope = ((total(h) - total(-h)) / (2 * h)).item()       # off by h^2 times a third derivative: about 1e-6 of it
    lse = reference(o)[1].float()
    got = backward(o, M, N, K, "bf16", lse, dloss=torch.ones(M, device="cuda"), smoothing=0.1, dx_dtype="f32", dw_dtype="f32")
    terms = [got["dx"].double() * dx, got["dw"].double() * dw, got["dbias"].double() * db]
    # every element carries at most bf16's half step of its terms, 2^-8 of twice the magnitudes of dz
    bound = sum((t.abs().sum().item() for t in terms)) * HALF * 2
    assert abs(sum(t.sum().item() for t in terms) - slope) <= bound + 1e-4 * abs(slope)


# ----------------------------------------------------------------------------- use

def test_equal_calls_give_equal_bits():
    for M, N, K in ((2, 1000, 256), (64, 1000, 4096), (2304, 4864, 64)):
        o = make(M, N, K, "bf16", seed=16)
        a, b = forward(o, M, N, K, "bf16"), forward(o, M, N, K, "bf16")
        assert all(torch.equal(p, q) for p, q in zip(a, b))
        d = torch.ones(M, device="cuda")
        p, q = backward(o, M, N, K, "bf16", a[1], dloss=d), backward(o, M, N, K, "bf16", a[1], dloss=d)
        assert all(torch.equal(p[k], q[k]) for k in p)


@pytest.mark.parametrize("M,N,K", [(2, 1000, 256), (64, 1000, 2048), (700, 1500, 128)])
def test_captured(M, N, K):
    """Forward and backward in a graph, replayed on other inputs between eager work."""
    s = step()
    desc = s.loss_desc(M, N, K, smoothing=0.1)
    held = make(M, N, K, "bf16", seed=17)
    loss, lse, mean = (torch.empty(n, device="cuda") for n in (M, M, 2))
    dmean = torch.ones(1, device="cuda")
    dx, dw, db = torch.empty_like(held["x"]), torch.empty_like(held["w"]), torch.empty(N, device="cuda")
    wf, wb = s.loss_workspace(desc), s.loss_workspace(desc, True)

    def call():
        s.fqt_loss_forward(desc, held["x"], held["w"], held["target"], loss, lse, wf, bias=held["bias"], mean=mean)
        s.fqt_loss_backward(desc, held["x"], held["w"], held["target"], lse, wb, dmean=dmean, mean=mean,
                            bias=held["bias"], dx=dx, dw=dw, dbias=db)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (18, 19, 20):
        o = make(M, N, K, "bf16", seed=seed)
        for k in ("x", "w", "target", "bias"):
            held[k].copy_(o[k])
        call()
        want = [t.clone() for t in (loss, lse, mean, dx, dw, db)]
        for t in (loss, lse, mean, dx, dw, db):
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (loss, lse, mean, dx, dw, db)))


def test_on_another_stream():
    M, N, K = 300, 700, 128
    o = make(M, N, K, "bf16", seed=21)
    want = forward(o, M, N, K, "bf16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = forward(o, M, N, K, "bf16")
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("smoothing", [0.0, 0.1])
def test_slopes_along_the_gradients(smoothing):
    """The slope of the float64 loss along the sign of each gradient by itself, where it is the sum of the gradient's magnitudes:
    dx and dw are off by 2^-8 of the magnitudes of their terms, dbias by its own float32."""
    M, N, K = 60, 90, 40
    o = make(M, N, K, "bf16", seed=25)
    z, lse64, _, counted, zerr, _ = reference(o, smoothing)
    got = backward(o, M, N, K, "bf16", lse64.float(), dloss=torch.ones(M, device="cuda"), smoothing=smoothing, dx_dtype="f32",
                   dw_dtype="f32")
    got = {k: v.double() for k, v in got.items()}
    p = torch.exp(z - lse64[:, None])
    q = torch.full_like(z, smoothing / N).scatter_add_(1, o["target"].clamp(min=0)[:, None],
                                                       torch.full_like(z[:, :1], 1 - smoothing))
    dz = (p + q) * counted[:, None]                         # at least the magnitudes
    off = {"dx": HALF * (dz @ o["w64"].abs()).sum(), "dw": HALF * (dz.t().contiguous() @ o["x64"].abs()).sum(), "dbias": 0.0}
    small = (600 * U + 4 * zerr.max() + (M + N) * U) * dz.sum() * (1 + o["x64"].abs().max() * K + o["w64"].abs().max() * K)
    h = 1e-4
    for name, key in (("dx", "x64"), ("dw", "w64"), ("dbias", "bias")):
        way = got[name].sign()

        def total(step):
            return reference(dict(o, **{key: o[key].double() + step * way}), smoothing)[2].sum()

        slope = (total(h) - total(-h)).item() / (2 * h)
        # (the difference itself: squares of h times the change of z, at most 1e-2, relative to the slope)
        bound = 2 * off[name] + (small if name != "dbias" else (600 * U + 4 * zerr.max() + M * U) * dz.sum()) + 1e-4 * slope
        assert slope > 0 and abs(got[name].abs().sum().item() - slope) <= bound, name
        assert bound < 0.1 * slope, name                    # that the bound says something


@pytest.mark.parametrize("M,N", [(2, 131072), (40, 131072), (600, 3000), (1500, 30011), (300, 700)])
@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_smoothed_sums_over_many_classes(M, N, kind):
    """The mean of z, all of it on one side of 0: at most N / 1024 + 160 additions one after the other, each off by u of the
    sum, and the roundings of z in units of log 2."""
    K = 16
    o = make(M, N, K, kind, seed=26, integers=True, ignored=0.0)
    o["bias"] = o["bias"] + 9.0
    loss, _, _ = forward(o, M, N, K, kind, 0.5)
    z, _, loss64, _, _, tail = reference(o, 0.5)
    big = z.abs().amax(dim=1)
    lim = 520 * U * tail + 8 * U * loss64.abs() + 0.5 * (N / 1024 + 160 + 16) * U * big
    err = (loss.double() - loss64).abs()
    assert (err <= lim).all(), f"loss off by {(err / lim).max().item():.3g} of the bound"
