"""The orthogonalised update with coefficients of its own for every step, in single steps and in groups of them.

The schedules are of the minimax kind: each polynomial is the best on the range that the ones before it leave, ends exactly at that
range's edge and is steep beyond it.  So what the kernels hold a matrix's singular values for decides how many bits are stored.

Tolerances.  In single steps what test_gpu_ortho.py allows: twice the error of the same formula in float32.  In groups of float32 sets
a rounding of A has grown by 200 at the most when it meets X, where X's own roundings have grown by sqrt(200) = 14 (A is X's square):
a few times the error of single steps in the mean, sixteen as a limit.  bfloat16 results: the group's error is below half a step's
mean, 2^-9, by four, 2^-11 of the norm; a value that falls on the other side of a tie for it is off by as much as the tie was and
twice that."""
import numpy as np
import pytest
import torch

from oracle import ops_oracle as orc
from test_gpu_ortho import EPS, QUINTIC, SHARP, gradient, large_set, run

pytestmark = pytest.mark.gpu

# singular values from 1e-3 on, by polynomials that were rounded to four digits; the second with two steps of the limit's behind it
MINIMAX = [(8.4703, -25.1081, 18.6293), (4.1828, -3.1087, 0.5806), (3.9619, -2.9541, 0.5630), (3.2866, -2.4647, 0.5074),
           (2.2737, -1.6447, 0.4162), (1.8887, -1.2652, 0.3765)]
STEEP = [(8.287, -23.596, 17.300), (4.107, -2.948, 0.5448), (3.949, -2.909, 0.5518), (3.318, -2.488, 0.5100), (2.3007, -1.6689, 0.4188),
         (1.8913, -1.2680, 0.3768), SHARP, SHARP]
MIXED = [(1.5, -0.5, 0.0), QUINTIC, (0.9, 0.3, -0.2), (2.0, -1.5, 0.5), (1.2, 0.0, -0.1), SHARP, (3.0, -3.0, 1.0)]
SCHEDULES = {"minimax": MINIMAX, "steep": STEEP, "mixed": MIXED}


def plain(G, coeffs):
    X = torch.from_numpy(G if G.shape[0] <= G.shape[1] else G.T.copy())
    X = X / (X.double().norm().float() + EPS)
    for a, b, c in coeffs:
        A = X @ X.T
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.double().numpy() if G.shape[0] <= G.shape[1] else X.double().numpy().T


def rounded(coeffs):
    return [tuple(float(np.float32(v)) for v in abc) for abc in coeffs]


def holds(mats, got, coeffs, times, which):
    for i in which:
        want = orc.orthogonalize(mats[i], rounded(coeffs), EPS)
        err, of_plain = np.linalg.norm(got[i] - want), np.linalg.norm(plain(mats[i], rounded(coeffs)) - want)
        assert err <= times * of_plain + 2.0 ** -24 * np.linalg.norm(want), (mats[i].shape, err, of_plain, np.linalg.norm(want))


def holds_in_bf16(mats, got, coeffs, which):
    for i in which:
        want = orc.orthogonalize(mats[i], rounded(coeffs), EPS)
        nearest = torch.from_numpy(want).to(torch.bfloat16).double().numpy()
        err, of_rounding = np.linalg.norm(got[i] - want), np.linalg.norm(nearest - want)
        assert err <= of_rounding + 2.0 ** -10 * np.linalg.norm(want), (mats[i].shape, err, of_rounding, np.linalg.norm(want))


@pytest.mark.parametrize("name", SCHEDULES)
@pytest.mark.parametrize("shape", [(512, 1024), (1024, 512), (200, 330)])
def test_single_steps(shape, name):
    for coeffs in (SCHEDULES[name], SCHEDULES[name][:3]):
        mats = [gradient(*shape, seed=1)]
        holds(mats, run(mats, coeffs), coeffs, 2, [0])
        holds_in_bf16(mats, run(mats, coeffs, "bf16"), coeffs, [0])


@pytest.mark.parametrize("tiles", [64, 128])
@pytest.mark.parametrize("name", SCHEDULES)
def test_groups_of_steps(name, tiles):
    # (a sum of m m n from 6e8 on that is 1.4 times that of m^3: groups; 192 tiles of 128 on and below the diagonals at the most: tiles of 64)
    sizes = [(512, 1024), (1000, 400), (390, 1030), (512, 900)] if tiles == 64 else [(512, 1024), (1000, 400), (390, 1030), (512, 900)] * 6
    mats = [gradient(r, c, i) for i, (r, c) in enumerate(sizes)]
    m = np.array([sorted(a.shape) for a in mats], dtype=np.float64)
    assert (m[:, 0] ** 2 * m[:, 1]).sum() >= max(6e8, 1.4 * (m[:, 0] ** 3).sum())
    assert (sum(t * (t + 1) // 2 for t in (-(-min(a.shape) // 128) for a in mats)) > 192) == (tiles == 128)
    for steps in (2, 4, len(SCHEDULES[name])):
        coeffs = SCHEDULES[name][:steps]
        holds(mats, run(mats, coeffs), coeffs, 16, range(4))
        holds_in_bf16(mats, run(mats, coeffs, "bf16"), coeffs, range(4))


def test_every_step_of_a_group_has_its_own_coefficients():
    """A set alone in single steps against the same matrices in groups: any two steps that changed places would show."""
    mats = [gradient(512, 1100, i) for i in range(4)]
    for first in range(3):
        coeffs = (MIXED + MIXED)[first:first + 6]
        grouped = run(mats, coeffs)
        for i in (0, 3):
            alone = run([mats[i]], coeffs)[0]
            assert np.linalg.norm(grouped[i] - alone) <= 2.0 ** -16 * np.linalg.norm(alone)
            swapped = orc.orthogonalize(mats[i], rounded([coeffs[1], coeffs[0]] + coeffs[2:]), EPS)
            assert np.linalg.norm(swapped - alone) > 2.0 ** -13 * np.linalg.norm(alone)


@pytest.mark.parametrize("name", ["minimax", "steep"])
def test_matrices_of_rank_one_stay_finite(name):
    """The gradient of an expert that saw one token: its singular value is 1 to the last bit, at the edge of every range."""
    rng = np.random.default_rng(5)
    for shape in ((96, 300), (700, 400)):
        G = np.outer(rng.normal(size=shape[0]), rng.normal(size=shape[1])).astype(np.float32)
        coeffs = SCHEDULES[name]
        holds([G], run([G], coeffs), coeffs, 2, [0])


@pytest.mark.parametrize("kind", ["long", "square"])
def test_bf16_results_of_large_sets_are_near_the_nearest(kind):
    """Wide, tall and odd ones, a matrix of one value and a narrow one among them."""
    mats = large_set(kind)
    for steps in (2, 5):
        holds_in_bf16(mats, run(mats, [QUINTIC] * steps, "bf16"), [QUINTIC] * steps,
                      (0, 1, 2, 3, 4, 6, len(mats) - 3, len(mats) - 2, len(mats) - 1))


def spectrum(kind, m=512, n=1024):
    rng = np.random.default_rng(8)
    if kind == "noise":
        return rng.normal(size=(m, n)).astype(np.float32)
    values = {"a hundredth": np.logspace(0, -2, m), "1e-4": np.logspace(0, -4, m), "one and many": np.r_[1.0, np.full(m - 1, 0.01)]}[kind]
    u, v = np.linalg.qr(rng.normal(size=(m, m)))[0], np.linalg.qr(rng.normal(size=(n, m)))[0]
    return ((u * values) @ v.T).astype(np.float32)


@pytest.mark.parametrize("name", ["minimax", "steep", "usual"])
def test_groups_are_near_float32_products_whatever_the_singular_values(name):
    """Four times the error of float32 products, as test_gpu_ortho.py allows groups."""
    coeffs = [QUINTIC] * 5 if name == "usual" else SCHEDULES[name]
    mats = [spectrum(k) for k in ("noise", "a hundredth", "1e-4", "one and many")] * 2
    holds(mats, run(mats, coeffs), coeffs, 4, range(4))
    holds_in_bf16(mats, run(mats, coeffs, "bf16"), coeffs, range(4))
