"""The row kernels of the training operators, from their CUDA sources, on the host: every copy within its matrix, nothing written
beside the outputs, no barrier misused, under random schedules; values against the definitions in 64 bits.

The cases are those that a GPU should not be the first to see: matrices that begin off 16 bytes, rows that overlap, many rows
a group with few groups, outputs over inputs."""
import pytest
import torch

import host_rows
import training_reference as ref

pytestmark = pytest.mark.skipif(host_rows.cuda_include() is None, reason="needs CUDA's headers")

KINDS = ("f32", "bf16")


@pytest.fixture(scope="session")
def libs(tmp_path_factory):
    return host_rows.build(str(tmp_path_factory.mktemp("rows")), [(f, k) for f in ("norm", "xent") for k in KINDS])


def given(n, d, dtype, ld, first, seed, scale, offset=0.0):
    """A matrix of random values; what lies between its rows is NaN.  (Overlapping rows: the last one written counts.)"""
    m = host_rows.Matrix(n, d, dtype, ld, first, float("nan"))
    values = torch.randn(n, d, generator=torch.Generator().manual_seed(seed)) * scale + offset
    for i in range(n):
        m.m[i] = values[i].to(dtype)
    return m


# rows, columns, row distance less columns (below 0: rows overlap; None: distance 0), first element, output (lies as the input
# does, or dense), clusters at most
CASES = [
    (1, 3, 0, 1, "same", 1), (7, 5, 0, 3, "same", 1), (90, 6, 1, 1, "same", 2), (40, 16, 0, 2, "same", 1), (65, 33, 0, 5, "same", 1),
    (50, 100, 4, 1, "same", 2), (50, 100, 3, 7, "same", 1), (30, 250, 0, 1, "same", 1), (21, 300, 8, 3, "same", 1),
    (21, 520, 0, 5, "same", 1), (13, 777, 0, 1, "same", 1), (17, 1000, 24, 4, "same", 1), (17, 1001, 0, 2, "same", 2),
    (9, 1500, 3, 1, "same", 1), (11, 2050, 0, 7, "same", 1), (19, 4100, 0, 1, "same", 2), (17, 4096, 0, 0, "same", 1),
    (12, 6200, 0, 3, "same", 1), (11, 9000, 5, 1, "same", 1), (11, 8200, 0, 0, "same", 1), (10, 16400, 0, 5, "same", 1),
    (10, 25003, 0, 0, "same", 1), (9, 33000, 0, 4, "same", 1), (13, 768, None, 1, "dense", 1), (6, 9001, None, 3, "dense", 1),
    (40, 64, None, 0, "dense", 1), (12, 700, -699, 0, "dense", 1), (12, 64, -60, 1, "dense", 1), (8, 2000, -1000, 3, "dense", 1),
    (24, 768, 13, 0, "dense", 1), (10, 5001, 0, 0, "dense", 1), (60, 40, 0, 1, "dense", 1),
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_rows(libs, case, kind):
    n, d, more, first, how, resident = case
    ld = 0 if more is None else d + more
    dtype = host_rows.TYPES[kind][0]
    lies = (ld, first) if how == "same" else (d, 0)
    seed = n * 7 + d
    norm, xent = libs["norm", kind], libs["xent", kind]
    x, dy = given(n, d, dtype, ld, first, seed, 1.0, 0.5), given(n, d, dtype, ld, first, seed + 1, 0.1)
    gen = torch.Generator().manual_seed(seed + 2)
    w, b = 1 + 0.2 * torch.randn(d, generator=gen), 0.2 * torch.randn(d, generator=gen)

    y, mean, rstd = host_rows.Matrix(n, d, dtype, *lies, 7.0), torch.empty(n), torch.empty(n)
    assert norm.layer_norm(x.m, w, b, y.m, mean, rstd, resident=resident, seed=seed) == 0 and norm.report == ""
    want, bound = ref.norm(x.m, w, b, 1e-5)
    for g, v, e, name in zip((y.m, mean, rstd), want, bound, ("y", "mean", "rstd")):
        ref.assert_within(g, v, e, name)
    assert y.kept()

    want, bound = ref.norm_grad(dy.m, x.m, mean, rstd, w, torch.float32)
    for need in ((1, 1, 1), (0, 1, 1), (1, 0, 0)):
        dx, dw, db = host_rows.Matrix(n, d, dtype, *lies, 7.0), torch.zeros(d), torch.zeros(d)
        outs = [o if k else None for o, k in zip((dx.m, dw, db), need)]
        assert norm.layer_norm_backward(dy.m, x.m, mean, rstd, w, *outs, resident=resident, seed=seed) == 0 and norm.report == ""
        for g, v, e, name in zip(outs, want, bound, ("dx", "dw", "db")):
            if g is not None:
                ref.assert_within(g, v, e, name)
        assert dx.kept()

    z = given(n, d, dtype, ld, first, seed + 3, 3.0)
    labels = torch.randint(0, d, (n,), generator=gen, dtype=torch.int32)
    labels[torch.rand(n, generator=gen) < 0.2] = -1
    want, bound = ref.cross_entropy(z.m, labels, True)
    for form in ("given", "none") + (("over",) if how == "same" else ()):
        loss, row = torch.zeros(()), torch.zeros(n)
        dz = None if form == "none" else z if form == "over" else host_rows.Matrix(n, d, dtype, *lies, 7.0)
        rc = xent.label_cross_entropy(z.m, labels, True, loss, row, None if dz is None else dz.m, resident=resident, seed=seed)
        assert rc == 0 and xent.report == ""
        for g, v, e, name in zip((loss, row, None if dz is None else dz.m), want, bound, ("loss", "row_loss", "dlogits")):
            if g is not None:
                ref.assert_within(g, v, e, name)
        assert dz is None or dz.kept()


# A copy that never lands, as no healthy run sees it: shapes of a warp, two, four and eight warps a row, and clusters of two, four
# and eight blocks; rows enough that the ring comes round after it.
LATE = [("f32", 60, 520, 5), ("f32", 40, 777, 9), ("f32", 40, 1000, 7), ("f32", 30, 1500, 6), ("f32", 30, 4096, 3), ("f32", 20, 6200, 2),
        ("f32", 18, 8200, 4), ("f32", 14, 16400, 9), ("f32", 12, 25003, 11), ("bf16", 90, 768, 30), ("bf16", 40, 1001, 11),
        ("bf16", 30, 4096, 5), ("bf16", 20, 9000, 3), ("bf16", 12, 24576, 12)]


def late_inputs(kind, n, d):
    dtype = host_rows.TYPES[kind][0]
    return given(n, d, dtype, d, 0, d, 1.0, 0.5).m, given(n, d, dtype, d, 0, d + 1, 0.1).m, dtype


def healthy_or_nan(got, want):
    """Rows of `got` that hold a NaN; every other element has to be what it is without the loss."""
    bad = got.isnan()
    assert torch.equal(got[~bad], want[~bad])
    rows = bad.any(1) if got.dim() > 1 else bad
    if got.dim() > 1:
        assert bad[rows].all()
    return rows


@pytest.mark.parametrize("kind,n,d,lost", LATE)
def test_a_copy_that_never_lands(libs, kind, n, d, lost):
    """Rows that depend on it are NaN, no barrier gets an arrival too many, no block ends while copies are on their way."""
    x, dy, dtype = late_inputs(kind, n, d)
    norm, xent = libs["norm", kind], libs["xent", kind]
    w, b = torch.ones(d), torch.zeros(d)
    got = []
    for k in (0, lost):
        y, mean, rstd = torch.zeros(n, d, dtype=dtype), torch.empty(n), torch.empty(n)
        assert norm.layer_norm(x, w, b, y, mean, rstd, resident=1, seed=d, lost=k) == 0 and norm.report == ""
        got.append((y, mean, rstd))
    rows = healthy_or_nan(got[1][0], got[0][0])
    assert rows.any() and torch.equal(healthy_or_nan(got[1][1], got[0][1]), rows) and torch.equal(healthy_or_nan(got[1][2], got[0][2]), rows)
    _, mean, rstd = got[0]
    got = []
    for k in (0, lost):
        dx, dw, db = torch.zeros(n, d, dtype=dtype), torch.zeros(d), torch.zeros(d)
        assert norm.layer_norm_backward(dy, x, mean, rstd, w, dx, dw, db, resident=1, seed=d, lost=k) == 0 and norm.report == ""
        got.append(dx)
    assert healthy_or_nan(got[1], got[0]).any()
    labels = (torch.arange(n) % d).to(torch.int32)
    got = []
    for k in (0, min(lost, n)):
        loss, row, dz = torch.zeros(()), torch.zeros(n), torch.zeros(n, d, dtype=dtype)
        assert xent.label_cross_entropy(x, labels, True, loss, row, dz, resident=1, seed=d, lost=k) == 0 and xent.report == ""
        got.append((loss, row, dz))
    rows = healthy_or_nan(got[1][2], got[0][2])
    assert rows.any() and torch.equal(healthy_or_nan(got[1][1], got[0][1]), rows) and got[1][0].isnan()


@pytest.mark.parametrize("kind,n,d,lost", [("f32", 20, 6200, 9), ("f32", 14, 24576, 300), ("f32", 12, 32768, 2000), ("bf16", 20, 9000, 100)])
def test_a_message_that_never_lands(libs, kind, n, d, lost):
    """What the cluster works out after it is NaN; nothing is wrong, and nothing waits for ever."""
    x, dy, dtype = late_inputs(kind, n, d)
    norm, xent = libs["norm", kind], libs["xent", kind]
    w, b = torch.ones(d), torch.zeros(d)
    labels = (torch.arange(n) % d).to(torch.int32)
    got = []
    for k in (0, lost):
        y, mean, rstd = torch.zeros(n, d, dtype=dtype), torch.empty(n), torch.empty(n)
        assert norm.layer_norm(x, w, b, y, mean, rstd, resident=1, seed=d, lost_message=k) == 0 and norm.report == ""
        if not got:
            stats = mean, rstd
        dx, dw, db = torch.zeros(n, d, dtype=dtype), torch.zeros(d), torch.zeros(d)
        assert norm.layer_norm_backward(dy, x, *stats, w, dx, dw, db, resident=1, seed=d, lost_message=k) == 0 and norm.report == ""
        loss, row, dz = torch.zeros(()), torch.zeros(n), torch.zeros(n, d, dtype=dtype)
        assert xent.label_cross_entropy(x, labels, True, loss, row, dz, resident=1, seed=d, lost_message=k) == 0 and xent.report == ""
        got.append((y, dx, dz, mean, rstd, row))
    for i, (a, c) in enumerate(zip(got[1], got[0])):
        bad = a.isnan()
        assert torch.equal(a[~bad], c[~bad]), i
        if i < 3:
            assert bad.any() and not bad.all(), i


@pytest.mark.parametrize("need_dx", [True, False])
@pytest.mark.parametrize("kind,n,d,lost", LATE)
def test_sums_over_rows_that_never_came(libs, kind, n, d, lost, need_dx):
    """The weight's and the bias's gradient are NaN in every column of which a row was lost, and right in the others."""
    x, dy, dtype = late_inputs(kind, n, d)
    norm = libs["norm", kind]
    mean, rstd = torch.full((n,), 0.5), torch.ones(n)
    w = torch.ones(d)
    want, bound = ref.norm_grad(dy, x, mean, rstd, w, torch.float32)
    dx, dw, db = torch.zeros(n, d, dtype=dtype) if need_dx else None, torch.zeros(d), torch.zeros(d)
    assert norm.layer_norm_backward(dy, x, mean, rstd, w, dx, dw, db, resident=1, seed=d, lost=lost) == 0 and norm.report == ""
    bad = dw.isnan()
    assert torch.equal(bad, db.isnan()) and bad.any()
    if d <= 4096:
        assert bad.all()                                  # one block a row
    for g, v, e in ((dw, want[1], bound[1]), (db, want[2], bound[2])):
        ref.assert_within(g[~bad], v[~bad], e[~bad])
