"""How the dense operators lay out their matrix products (host only): every accepted size can be launched."""
import pytest

torch = pytest.importorskip("torch")
fqt = pytest.importorskip("paper_2408_14267_amd.fqt", reason="libfqt.so not built")
from paper_2408_14267_amd import dense  # noqa: E402


def launches(p):
    return [(p.tile[i], p.threads[i], p.workgroups[i]) for i in range(p.launches)]


def covers(p, rows, cols, symmetric=False):
    """Whether the workgroups of a plan's launches are those of its tiles: all of one edge, or Large tiles
    with the last ones as sixteenths."""
    def tiles(b):
        m, n = -(-rows // b), -(-cols // b)
        return m * (m + 1) // 2 if symmetric else m * n
    (edge, _, first), *rest = launches(p)
    if not rest:
        return first == tiles(edge) * p.splits
    return p.splits == 1 and edge == 256 and rest[0][0] == 64 and first + rest[0][2] // 16 == tiles(256)


@pytest.mark.parametrize("M,N,K", [(1 << 30, 1, 8), (1 << 30, 64, 8), ((1 << 31) - 257, 1, 1), (5, 1 << 22, 1 << 16),
                                   (1 << 20, 1 << 18, 64), (1 << 19, 1 << 19, 1 << 19), (1 << 24, 16, 1 << 13),
                                   (7, 3, 1 << 22)])
@pytest.mark.parametrize("xt", ["bf16", "int8", "e4m3"])
def test_largest_sizes_are_launchable(M, N, K, xt):
    """A launch counts its threads in 32 bits: 2^30 rows of one column are 2^24 tiles of 64 x 64, 2^32 threads."""
    if xt == "int8" and K > 133144:
        K = 133144
    d = dense.linear_desc(M, N, K, x_dtype=xt)
    assert dense.fqt_linear_workspace_size(d) and dense.fqt_linear_workspace_size(d, True)
    for product, rows, cols in (("forward", M, N), ("dx", M, K), ("dw", N, K)):
        p = dense.fqt_linear_plan(d, product)
        assert p.launches in (1, 2) and covers(p, rows, cols), launches(p)
        assert all(t * w < 1 << 32 for _, t, w in launches(p)), launches(p)


@pytest.mark.parametrize("M,N,K", [((1 << 31) - 1, 1, 1), (1 << 30, 1, 513), (1 << 20, 1 << 19, 64), (4, 1 << 22, 1 << 17)])
def test_sizes_past_one_launch_are_refused(M, N, K):
    d = dense.linear_desc(M, N, K)
    for call in (lambda: dense.fqt_linear_workspace_size(d), lambda: dense.fqt_linear_workspace_size(d, True),
                 lambda: dense.fqt_linear_plan(d)):
        with pytest.raises(fqt.FqtError) as e:
            call()
        assert e.value.status == fqt.FQT_E_SHAPE


@pytest.mark.parametrize("rows,cols", [(65536, 262136), (262143, 65528), (65, (1 << 22) - 1), (4096, 25088), (512, 4608)])
def test_orthogonalisations_are_launchable(rows, cols):
    d = dense.ortho_desc(rows, cols)
    m, n = -(-min(rows, cols) // 64) * 64, -(-max(rows, cols) // 64) * 64
    for product in dense.ORTHO_PRODUCTS:
        p = dense.fqt_ortho_plan(d, product)
        assert covers(p, m, n if product == "apply" else m, product != "apply"), launches(p)
        assert all(t * w < 1 << 32 for _, t, w in launches(p))


def test_plan_refusals():
    d, o, p = dense.linear_desc(8, 16, 32), dense.ortho_desc(100, 200), dense.fqt_product_plan()
    lib = dense._lib
    assert lib.fqt_linear_plan(d, 3, p) == lib.fqt_ortho_plan(o, -1, p) == fqt.FQT_E_INVAL
    assert lib.fqt_linear_plan(d, 0, None) == lib.fqt_ortho_plan(o, 0, None) == fqt.FQT_E_NULL
    assert lib.fqt_linear_plan(None, 0, p) == lib.fqt_ortho_plan(None, 0, p) == fqt.FQT_E_NULL
    with pytest.raises(ValueError, match="unknown product"):
        dense.fqt_linear_plan(d, "gram")
    assert dense.fqt_linear_plan(dense.linear_desc(4, 16, 32)).launches == 0       # the few-row form
    assert dense.fqt_ortho_plan(dense.ortho_desc(64, 200), "gram").launches == 0
