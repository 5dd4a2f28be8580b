"""Pins of the oracle of the operations on compact targets: worked cases, the theorem of
speculative sampling, and the oracle of verification from logits."""
from fractions import Fraction

import numpy as np
import pytest

import oracle
from oracle import compact


def _softmax(x):
    e = np.exp(x - x.max(-1, keepdims=True))
    return (e / e.sum(-1, keepdims=True)).astype(np.float32)


def test_units_round_to_nearest():
    for x in (0.0, 1.0, 0.1, 2.0 ** -62, 2.0 ** -63, 3 * 2.0 ** -63, 1.9999999):
        want = round(Fraction(float(np.float32(x))) * 2 ** 62)  # Python rounds ties to even, too
        assert int(compact.units(np.float32([x]))[0]) == want


def test_worked_verify_probs():
    """V = 4, dyadic probabilities: every product and sum below is exact."""
    p = np.float32([[[0.25, 0.25, 0.5, 0.0], [0.125, 0.125, 0.25, 0.5]]])
    q = np.float32([[[0.5, 0.5, 0.0, 0.0]]])
    one = lambda y, u0, u1, q=q, **kw: tuple(x.tolist() for x in compact.verify_probs(q, p, [[y]], [[u0, u1]], **kw))
    # p/q = 1/2 at token 0: accepted below it, strictly; the residual is (0, 0, 1/2, 0)
    assert one(0, 0.49, 0.6) == ([1], [[0, 3]], [[0]])
    assert one(0, 0.5, 0.0) == ([0], [[2, -1]], [[1]])
    # the bonus row's prefix sums are 1/8, 1/4, 1/2, 1: min{ j : C_j > u }
    for u, j in ((0.0, 0), (0.125, 1), (0.2, 1), (0.25, 2), (0.5, 3), (0.99, 3)):
        assert one(0, 0.0, u) == ([1], [[0, j]], [[0]])
    # no drafts at all: the draw is from row 0 (sums 1/4, 1/2, 1, 1)
    assert one(-1, 0.0, 0.25, lens=[0]) == ([0], [[1, -1]], [[0]])
    assert one(-1, 0.0, 0.999, lens=[0]) == ([0], [[2, -1]], [[0]])
    # a certain proposal: accepted with probability p(y); the residual is p without y
    assert one(2, 0.49, 0.3, q=None) == ([1], [[2, 2]], [[0]])
    assert one(2, 0.5, 0.49, q=None) == ([0], [[0, -1]], [[1]])
    assert one(2, 0.5, 0.5, q=None) == ([0], [[1, -1]], [[1]])
    # p(y) = 0 never passes; q(y) = 0 < p(y) always does
    assert one(3, 0.0, 0.0)[0] == [0]
    assert one(2, 0.999, 0.0)[0] == [1]
    # bad token, bad length
    assert one(4, 0.0, 0.0) == ([-1], [[-1, -1]], [[0]])
    assert one(0, 0.0, 0.0, lens=[2]) == ([-1], [[-1, -1]], [[0]])


def test_no_weight_left_takes_the_first_maximum():
    p, q = np.float32([[[0.1, 0.2, 0.2, 0.1], [1, 0, 0, 0]]]), np.float32([[[0.2, 0.4, 0.2, 0.2]]])
    acc, out, mask = compact.verify_probs(q, p, [[1]], [[0.75, 0.3]])
    assert acc[0] == 0 and out.tolist() == [[1, -1]] and mask.tolist() == [[1]]


@pytest.mark.parametrize("certain", [False, True])
def test_every_emitted_token_is_distributed_as_p(certain):
    """The theorem of speculative sampling (Section 3), by a chi-square test at a fixed seed."""
    rng = np.random.default_rng(5)
    V, N = 5, 40000
    p, q = _softmax(rng.normal(size=V)), _softmax(rng.normal(size=V))
    y = np.full(N, 2) if certain else rng.choice(V, size=N, p=q.astype(np.float64) / q.astype(np.float64).sum())
    u = rng.random((N, 2), dtype=np.float32)
    rows = np.broadcast_to(p, (N, 2, V))
    _, out, _ = compact.verify_probs(None if certain else np.broadcast_to(q, (N, 1, V)), rows, y[:, None], u)
    count = np.bincount(out[:, 0], minlength=V)
    chi2 = ((count - N * p) ** 2 / (N * p)).sum()
    assert chi2 < 23.5  # 4 degrees of freedom: P(chi2 > 23.5) = 1e-4


@pytest.mark.parametrize("T", [1.0, 0.7])
def test_agrees_with_verification_from_logits(T):
    """Where p and q are the softmax of the logits, the decisions are those of the oracle of
    verification from logits, wherever its margins exceed the rounding of p and q to fp32."""
    rng = np.random.default_rng(6)
    B, k, V = 200, 4, 37
    z = rng.normal(size=(B, k, V)).astype(np.float32)
    t = np.concatenate([z + rng.normal(size=z.shape).astype(np.float32) * 0.7, z[:, :1]], 1)
    y, u = rng.integers(0, V, (B, k)).astype(np.int32), rng.random((B, k + 1), dtype=np.float32)
    ref = oracle.verify(z, t, y, u, T)
    acc, out, mask = compact.verify_probs(_softmax(z / T), _softmax(t / T), y, u)
    clear = (np.nan_to_num(ref["margin"], nan=1.0).min(1) > 1e-4) & (np.nan_to_num(ref["cdf_gap"], nan=1.0) > 1e-5)
    assert clear.sum() > 150
    assert np.array_equal(acc[clear], ref["accepted"][clear])
    assert np.array_equal(out[clear], ref["out_tokens"][clear])
    assert np.array_equal(mask[clear], ref["mismatch_mask"][clear])


# ------------------------------------------------------------------ top logits
def test_worked_topk():
    x = np.float32([[1, 3, 3, -np.inf, 0, 3, -0.0], [-np.inf, -np.inf, 2, -np.inf, -np.inf, -np.inf, -np.inf]])
    v, i, r = compact.topk(x, 4, 0.5)
    assert i.tolist() == [[1, 2, 5, 0], [2, 0, 1, 3]]
    assert v.tolist() == [[3, 3, 3, 1], [2, -np.inf, -np.inf, -np.inf]]
    assert r[0] == pytest.approx(np.log(2.0)) and r[1] == -np.inf
    assert compact.topk(x, 7)[2].tolist() == [-np.inf, -np.inf]


def test_topk_and_its_rest_make_up_the_row():
    rng = np.random.default_rng(2)
    x = rng.normal(size=(50, 301)) * 4
    for tau in (0.5, 1.0, 2.0):
        v, i, r = compact.topk(x, 20, tau)
        total = np.logaddexp(np.log(np.exp(v / tau).sum(1)), r)
        np.testing.assert_allclose(total, np.log(np.exp(x / tau).sum(1)), rtol=1e-13)
        assert (np.diff(v, axis=1) <= 0).all() and np.array_equal(np.sort(x, axis=1)[:, ::-1][:, :20], v)


# ------------------------------------------------------------------ distillation from top logits
KINDS = ["fkl", "rkl", "jsd", "tvd", "ce"]


def _case(seed, V=9, K=4, rest=True):
    rng = np.random.default_rng(seed)
    z, t = rng.normal(size=V) * 2, rng.normal(size=(1, V)) * 2
    v, i, r = compact.topk(t, K, 1.0)
    return z, v[0], i[0], (r[0] if rest else None)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0])
def test_gradient_against_differences(kind, tau):
    for seed in range(6):
        z, v, i, r = _case(seed)
        if seed == 5:
            i = np.where(np.arange(len(i)) == 1, -1, i)  # an unused entry: its token joins the others
        loss, grad, _, _ = compact.distill_topk_row(z, v, i, r, kind, 0.3, tau)
        for j in range(len(z)):
            h = 1e-5
            up, dn = z.copy(), z.copy()
            up[j] += h
            dn[j] -= h
            d = (compact.distill_topk_row(up, v, i, r, kind, 0.3, tau)[0] -
                 compact.distill_topk_row(dn, v, i, r, kind, 0.3, tau)[0]) / (2 * h)
            assert grad[j] == pytest.approx(d, abs=1e-8)


@pytest.mark.parametrize("kind", KINDS)
def test_all_entries_kept_is_the_full_distillation(kind):
    rng = np.random.default_rng(3)
    z, t = rng.normal(size=(8, 11)) * 2, rng.normal(size=(8, 11)) * 2
    for tau in (0.7, 1.0):
        v, i, r = compact.topk(t, 11, tau)
        assert (r == -np.inf).all()
        loss, grad, _, _ = compact.distill_topk(z, v, i, r, kind, 0.3, tau)
        ref_l, ref_g = oracle.distill(z, t, None, kind, 0.3, temperature=tau)
        np.testing.assert_allclose(loss, ref_l, rtol=1e-10, atol=1e-12)
        np.testing.assert_allclose(grad, ref_g, rtol=1e-9, atol=1e-12)


def test_worked_distill_topk():
    """Masses in quarters: p = (1/2, 1/4 | 1/4), q = (1/4, 1/4 | 1/4 + 1/4)."""
    z, v, i = np.zeros(4), np.log([2.0, 1.0]), [2, 0]
    row = lambda kind, rest=np.log(1.0), **kw: compact.distill_topk_row(z, v, i, rest, kind, **kw)
    ln2 = np.log(2.0)
    assert row("fkl")[0] == pytest.approx(0.5 * ln2 - 0.25 * ln2)
    np.testing.assert_allclose(row("fkl")[1], [0, 0.125, -0.25, 0.125], atol=1e-15)
    assert row("rkl")[0] == pytest.approx(-0.25 * ln2 + 0.5 * ln2)
    assert row("tvd")[0] == pytest.approx(0.25)
    assert row("ce")[0] == pytest.approx(2 * ln2)
    # teacher cut to its kept tokens: p = (2/3, 1/3)
    assert row("fkl", None)[0] == pytest.approx(2 / 3 * np.log(8 / 3) + 1 / 3 * np.log(4 / 3))
    assert row("rkl", None)[0] == np.inf
    # no target mass, a repeated id, an id past the row
    assert row("jsd", -np.inf, beta=0.0)[0] == 0.0
    assert compact.distill_topk_row(z, v, [-1, -1], None, "fkl")[0] == 0.0
    assert np.isnan(compact.distill_topk_row(z, v, [2, 2], 0.0, "fkl")[0])
    assert np.isnan(compact.distill_topk_row(z, v, [2, 4], 0.0, "fkl")[0])


def test_bucketing_never_raises_a_divergence():
    """Merging the other tokens into one class loses information: f-divergences cannot grow."""
    rng = np.random.default_rng(4)
    z, t = rng.normal(size=(40, 30)) * 2, rng.normal(size=(40, 30)) * 2
    v, i, r = compact.topk(t, 6)
    for kind in ("fkl", "rkl", "jsd", "tvd"):
        full = oracle.distill(z, t, None, kind, 0.4)[0]
        cut = compact.distill_topk(z, v, i, r, kind, 0.4)
        assert (cut[0] <= full + 1e-12).all() and (cut[0] >= 0).all()
        np.testing.assert_allclose(cut[1].sum(1), 0, atol=1e-12)  # shift invariance
