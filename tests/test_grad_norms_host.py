"""The checks of gradients' norms see what they are for: gradients rounded as the kernels round
them pass, and ones with a mistake (planted here, in fp64) do not."""
import numpy as np
import pytest

from grad_norms import check_along, check_norm, gradient_errors
from oracle import doc_attention as oda

torch = pytest.importorskip("torch")

TYPES = {"bf16": (torch.bfloat16, 2.0 ** -8, 0.0), "f16": (torch.float16, 2.0 ** -11, 2.0 ** -25)}


def _rounded(x, dtype):
    return torch.tensor(x).float().to(TYPES[dtype][0]).double().numpy()


def _rounded_far(x, dtype, axis):
    """Rounded with the largest along axis near 2^10: as exact as the type is, however small."""
    top = np.abs(x).max(axis=axis, keepdims=True)
    f = 2.0 ** (10 - np.floor(np.log2(np.where(top > 0, top, 1.0))))
    return _rounded(x * f, dtype) / f


def _case(dtype, n, m, D, sharp, size, cap=0.0, mistake=""):
    rng = np.random.default_rng(1)
    q, k, v, do = (_rounded(rng.standard_normal((r, 1, D)) * s, dtype)
                   for r, s in ((n, sharp), (m, 1.0), (m, 1.0), (n, size)))
    sc, (_, u, tiny) = oda.Scores(None, cap), TYPES[dtype]
    s, t, _ = oda._head(q[:, 0], k[:, 0], sc, 0, 0)
    p, _ = oda._weights(s)
    dp = do[:, 0] @ v[:, 0].T
    o = _rounded(p @ v[:, 0], dtype)
    delta = (do[:, 0] * o).sum(axis=1, keepdims=True) if mistake == "D of the rounded output" else (p * dp).sum(axis=1, keepdims=True)
    ds = p * (dp - delta) * (1 - t * t)
    if mistake == "small numbers rounded as they are":
        a = b = _rounded(ds, dtype)
    else:
        a, b = _rounded_far(ds, dtype, 1), _rounded_far(ds, dtype, 0)
    scale = D ** -0.5
    got = [_rounded(x, dtype)[:, None] for x in (scale * a @ k[:, 0], scale * b.T @ q[:, 0], _rounded_far(p, dtype, 0).T @ do[:, 0])]
    if mistake == "the other sign":
        got = [-x for x in got]
    if mistake == "nothing":
        got = [0 * x for x in got]
    return got, gradient_errors(q, k, v, do, sc, 0, u, tiny)


CASES = [("bf16", 200, 200, 128, 20.0, 1.0, 0.0), ("f16", 40, 40, 64, 4.0, 1.0, 0.0), ("f16", 200, 3000, 64, 1.0, 1e-3, 0.0),
         ("f16", 200, 3000, 64, 1.0, 1e-4, 5.0), ("bf16", 300, 700, 64, 1.0, 1.0, 8.0)]


@pytest.mark.parametrize("case", CASES)
def test_rounded_gradients_pass(case):
    got, (want, error) = _case(*case)
    for name, x, y, e in zip(("dq", "dk", "dv"), got, want, error):
        check_norm(x, y, e, name)
        check_along(x, y, e, np.linalg.norm(y), name)


@pytest.mark.parametrize("case, mistake", [(CASES[0], "D of the rounded output"), (CASES[1], "D of the rounded output"),
                                           (CASES[2], "small numbers rounded as they are"),
                                           (CASES[3], "small numbers rounded as they are")])
def test_a_missing_part_fails(case, mistake):
    got, (want, error) = _case(*case, mistake=mistake)
    for i in (0, 1):
        with pytest.raises(AssertionError):
            check_norm(got[i], want[i], error[i], "")


@pytest.mark.parametrize("mistake", ["the other sign", "nothing"])
def test_wrong_directions_fail(mistake):
    for case in CASES:
        got, (want, error) = _case(*case, mistake=mistake)
        for x, y, e in zip(got, want, error):
            with pytest.raises(AssertionError):
                check_norm(x, y, e, "")
            with pytest.raises(AssertionError):
                check_along(x, y, e, np.linalg.norm(y), "")
