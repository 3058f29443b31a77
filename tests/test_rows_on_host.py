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
