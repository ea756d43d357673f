"""Pins of the oracle's distillation where the teacher's named tokens do not hold a mass of 1 minus the others': its gradient against
central differences of its own loss."""
import numpy as np
import pytest

from oracle import packed_ops as P
from test_oracle_packed_ops import differences

TAU = 1.5


def named_logits(rng, ids, mass):
    """Logits of a teacher whose log-sum-exp is 0 and whose entries hold so much of its mass (None: one of its own, 1)."""
    u = rng.standard_normal(ids.shape)
    return u if mass is None else u - TAU * np.log(np.exp(u / TAU).sum(axis=1, keepdims=True) / mass)


@pytest.mark.parametrize("mass", [None, 0.3, 0.7, 1.0, 1.04, 1.3])
@pytest.mark.parametrize("others", ["there", "masked", "none", "some masked"])
@pytest.mark.parametrize("twice", [False, True])
def test_gradient_is_the_losses(mass, others, twice):
    rng = np.random.default_rng(7)
    T, V, K = 4, 9, 9 if others == "none" else 4
    z, w = rng.standard_normal((T, V)), rng.random(T) + 0.1
    ids = np.argsort(rng.random((T, V)))[:, :K]
    if twice:
        ids = np.concatenate([ids, ids[:, :2]], axis=1)
    u = named_logits(rng, ids, mass)
    free = np.ones((T, V), bool)
    np.put_along_axis(free, ids, False, axis=1)
    if others == "masked":
        z[free] = -np.inf
    elif others == "some masked":
        z[np.arange(T), free.argmax(axis=1)] = -np.inf
    lse = None if mass is None else np.zeros(T)
    loss, total, dz = P.distill_loss(z, u, ids, lse, TAU, w)
    assert np.isfinite(loss).all() and np.isclose(total, np.sum(w * loss))
    with np.errstate(invalid="ignore"):
        want = differences(lambda x: P.distill_loss(x, u, ids, lse, TAU, w)[1], z)
    # second differences of the loss are below 1: an error of eps^2 / 6 and of rounding / eps
    assert np.allclose(dz, want, rtol=0, atol=1e-8)
    assert np.allclose(dz.sum(axis=1), 0, atol=1e-12)              # the loss does not change with all logits alike
