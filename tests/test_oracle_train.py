"""Pins of the checker's training operators: the loss on stored logits is Eq. 4's on whole rows when everything is stored,
gradients are those of differences."""
import numpy as np
import pytest

from oracle import cascade_oracle as O
from oracle import paged_oracle as PO
from oracle import train_oracle as TO


def _rows(seed, K=5, V=23, h=6):
    rng = np.random.default_rng(seed)
    return rng.normal(0, 2, (K, V)), rng.normal(0, 2, (K, V)), rng.standard_normal((K, h)), rng


def test_everything_stored_is_the_loss_on_whole_rows():
    target, draft, feat, rng = _rows(1)
    ids = np.stack([rng.permutation(target.shape[1]) for _ in target])
    top = np.take_along_axis(target, ids, 1)
    per, w, _ = O.drafter_loss(target, draft, feat, 0.1, 2.0)
    loss, saved, _ = TO.distill_loss(draft, top, ids, feat=feat, tau=0.1, c=2.0)
    assert np.allclose(loss, per, atol=1e-12) and np.array_equal(saved[:, 3], w) and np.allclose(saved[:, 2], 1.0)
    # with the rows' own log-sum-exp nothing changes either
    lse = np.log(np.exp(target).sum(1))
    assert np.allclose(TO.distill_loss(draft, top, ids, target_lse=lse, feat=feat, tau=0.1, c=2.0)[0], per, atol=1e-12)


def test_truncated_rows_are_the_loss_on_rows_truncated_to_minus_infinity():
    target, draft, feat, _ = _rows(2)
    ids = np.argsort(-target, 1)[:, :7]
    top = np.take_along_axis(target, ids, 1)
    cut = np.full_like(target, -np.inf)
    np.put_along_axis(cut, ids, top, 1)
    with np.errstate(invalid="ignore"):
        per = O.drafter_loss(cut, draft, feat, 2.0, 2.0)[0]
    assert np.allclose(TO.distill_loss(draft, top, ids)[0], per, atol=1e-12)


def test_sequences_and_padding():
    target, draft, feat, _ = _rows(3)
    feat = np.ones_like(feat)                                     # every pair converges
    ids, seq = np.argsort(-target, 1)[:, :4], np.array([0, 0, 1, -1, 2])
    top = np.take_along_axis(target, ids, 1)
    loss, saved, _ = TO.distill_loss(draft, top, ids, feat=feat, seq=seq)
    assert saved[:, 3].tolist() == [2.0, 1.0, 1.0, 0.0, 1.0] and loss[3] == 0
    assert not TO.distill_grad(draft, top, ids, saved)[3].any()


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("temperature", [1.0, 0.7])
def test_gradient_of_the_loss_by_differences(given, temperature):
    target, draft, feat, rng = _rows(4)
    ids = np.argsort(-target, 1)[:, :6].copy()
    top = np.take_along_axis(target, ids, 1)
    ids[0, 2], ids[1, 3], ids[2] = ids[0, 1], -1, -1              # a token twice, a place without an entry, none at all
    lse = np.log(np.exp(target / temperature).sum(1)) if given else None
    kw = dict(target_lse=lse, feat=feat, temperature=temperature, tau=0.0)
    up = rng.normal(0, 1, len(draft))
    grad = TO.distill_grad(draft, top, ids, TO.distill_loss(draft, top, ids, **kw)[1], up, 0.3, temperature)
    for _ in range(20):
        way, e = rng.standard_normal(draft.shape), 1e-5
        a, b = (TO.distill_loss(draft + s * e * way, top, ids, **kw)[0] for s in (1, -1))
        assert abs((up * (a - b)).sum() / (2 * e) * 0.3 - (grad * way).sum()) < 1e-8
    assert not grad[2].any()


@pytest.mark.parametrize("n,kv,Hq,Hkv,window,sinks", [(5, 5, 2, 2, 0, 0), (4, 9, 4, 2, 0, 0), (6, 11, 3, 1, 3, 2), (5, 3, 2, 1, 0, 0), (1, 1, 1, 1, 0, 0)])
def test_gradient_of_the_attention_by_differences(n, kv, Hq, Hkv, window, sinks):
    rng = np.random.default_rng(n + kv)
    D, scale = 4, 0.6
    x = [rng.standard_normal(s) for s in ((n, Hq, D), (kv, Hkv, D), (kv, Hkv, D))]
    up = rng.standard_normal((n, Hq, D))
    grads, sizes = TO.attention_grad(*x, up, window, sinks, scale)
    out, lse = PO.attention(*x, window, sinks, scale)
    again, _ = TO.attention_grad(*x, up, window, sinks, scale, out=out, lse=lse)
    for i in range(3):
        assert np.allclose(grads[i], again[i], atol=1e-12) and (np.abs(grads[i]) <= sizes[i] + 1e-12).all()
        for _ in range(5):
            way, e = rng.standard_normal(x[i].shape), 1e-5
            f = [(PO.attention(*[t + s * e * way if j == i else t for j, t in enumerate(x)], window, sinks, scale)[0] * up).sum() for s in (1, -1)]
            assert abs((f[0] - f[1]) / (2 * e) - (grads[i] * way).sum()) < 1e-7
