"""GPU: the loss from stored logits and its gradient where weights vanish and values are no numbers."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as TO
from paper_2605_07230_b200 import binding as cb
from tests import gpu_util as G
from tests.test_gpu_distill import Step, check_grad, check_loss, dev, make

pytestmark = pytest.mark.gpu

FEW, MANY = 3, 700                                                   # rows shared out over several blocks, and a block each


def falling(rng, K, V, n, T, gap):
    """Rows whose stored logits fall from entry to entry, the last of them `gap` (over T) below the first; the drafter leaves the
    last one's token out."""
    ids = np.stack([rng.permutation(V)[:n] for _ in range(K)]).astype(np.int32)
    top = np.repeat((-np.linspace(0, 1, n) ** 3 * gap * T).astype(np.float32)[None], K, 0)
    draft = rng.normal(0, 2 * T, (K, V)).astype(np.float32)
    draft[np.arange(K), ids[:, -1]] = -np.inf
    return draft, top, ids


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [FEW, MANY])
@pytest.mark.parametrize("T", [0.05, 1.0])
@pytest.mark.parametrize("V,n", [(16384, 64), (16384, 2000), (40001, 9)])
def test_an_entry_without_weight_at_a_logit_of_minus_infinity(V, n, T, K, dtype):
    """The gap lies past what 64 bits hold: the entry weighs nothing by any count."""
    draft, top, ids = falling(np.random.default_rng(n), K, V, n, T, 900.0)
    s = Step(draft, top, ids, dtype, temperature=T)
    s.forward()
    with np.errstate(invalid="ignore"):
        check_loss(s, TO.distill_loss(s.host, top, ids, temperature=T), T)
    assert s.loss.isfinite().all() and s.total.isfinite().all()


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("gap", [70.0, 84.0, 90.0, 140.0, 200.0])
def test_which_entries_weigh_something_does_not_depend_on_the_number_of_rows(gap, given):
    """Weights of 2^-101 and 2^-121, and what lies below 2^-126 and counts as none."""
    V, n, T = 16384, 64, 1.0
    draft, top, ids = falling(np.random.default_rng(5), MANY, V, n, T, gap)
    lse = np.full(MANY, np.log(np.exp(top[0].astype(np.float64)).sum()), np.float32) if given else None
    losses = []
    for K in (FEW, MANY):
        s = Step(draft[:K], top[:K], ids[:K], target_lse=None if lse is None else lse[:K])
        s.forward()
        losses.append(s.loss[:FEW].cpu().numpy())
    weighs = gap < 87                                                # 126 ln 2 = 87.3, with the log-sum-exp (2.6) in front or not
    assert not np.isnan(losses).any() and (np.isinf(losses) == weighs).all(), losses


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [500, 65536])
def test_a_position_without_weight_has_a_gradient_of_zeros_whatever_its_logits_hold(V, dtype):
    K, n = 5, 50
    _, draft, top, ids, _, _ = make(21, K, V, n)
    ids[0], top[1], ids[2] = -1, -np.inf, V
    draft[0, 7], draft[1, V - 1], draft[2, 3], draft[3, 4] = np.nan, np.inf, -np.inf, np.nan
    s = Step(draft, top, ids, dtype)
    s.forward()
    assert not s.loss[:3].any() and s.loss[3].isnan() and s.loss[4] > 0
    s.backward()
    assert not s.grad[:3].any() and not s.grad[:3].isnan().any() and s.grad[3].isnan().all()
    check_grad_row = TO.distill_grad(s.host[4:], top[4:], ids[4:], s.saved[4:].cpu().numpy())
    # p and q are off by at most 2^-18 here (exponents of at most 30 with two roundings), and rounded once
    assert np.abs(s.grad[4:].float().cpu().numpy() - check_grad_row).max() <= np.abs(check_grad_row).max() * (2.0**-8 + 2.0**-18)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("up", [np.nan, np.inf])
def test_padding_has_a_gradient_of_zeros_whatever_comes_back_from_above(up, dtype):
    K, V = 6, 3001
    _, draft, top, ids, _, _ = make(22, K, V, 30)
    draft[2] = np.nan
    seq, back = np.array([0, 0, -1, -1, 1, 1]), np.array([1.0, 0.5, up, up, 2.0, up], np.float32)
    s = Step(draft, top, ids, dtype, seq=seq)
    s.forward()
    s.backward(grad_loss=dev(back))
    assert not s.grad[2:4].any() and not s.grad[2:4].isnan().any()
    assert s.grad[[0, 1, 4]].isfinite().all() and not s.grad[5].isfinite().all()
    whole = s.host, s.grad, s.top, s.ids
    s.host, s.grad, s.top, s.ids = s.host[:2], s.grad[:2], s.top[:2], s.ids[:2]
    check_grad(s, s.saved[:2].cpu().numpy(), back[:2], 1.0, dtype=dtype)
    s.host, s.grad, s.top, s.ids = whole


@pytest.mark.parametrize("h", [8, 33])
def test_hidden_states_without_a_direction_do_not_converge(h):
    """Infinities, values that are no numbers, zeros: their cosine is no number."""
    K, V, n = 12, 200, 10
    _, draft, top, ids, _, rng = make(23, K, V, n)
    feat = np.repeat(rng.standard_normal((1, h)), K, 0).astype(np.float32)
    feat[1, 3], feat[4, 0], feat[6, 2], feat[9] = np.inf, -np.inf, np.nan, 0.0
    for tau in (-0.5, 0.5):
        s = Step(draft, top, ids, feat=feat, tau_seq=tau, c=3.0)
        s.forward()
        with np.errstate(invalid="ignore"):
            ref = TO.distill_loss(s.host, top, ids, feat=feat, tau=tau, c=3.0)
        assert ref[1][:, 3].tolist() == [1, 1, 3, 1, 1, 1, 1, 3, 1, 1, 3, 1]
        check_loss(s, ref)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K,V", [(7, 1003), (300, 65), (1, 129)])
def test_gradient_rows_between_the_logits_rows(K, V, dtype):
    """Logits and gradients as halves of one buffer's rows, either first."""
    _, draft, top, ids, _, _ = make(24, K, V, 20)
    for first in (0, 1):
        s = Step(draft, top, ids, dtype)
        rows = torch.full((K, 2, V + 3), float("nan"), device=G.DEV, dtype=s.draft.dtype)
        rows[:, first, :V] = s.draft
        s.draft, s.grad = rows[:, first, :V], rows[:, 1 - first, :V]
        s.forward()
        s.backward()
        check_grad(s, s.saved.cpu().numpy(), None, 1.0, dtype=dtype)
        assert np.array_equal(s.draft.float().cpu().numpy(), s.host) and rows[:, :, V:].isnan().all()
    with pytest.raises(cb.CascadeError):                             # by one element into the logits
        cb.cascade_distill_grad(rows[:, 0, :V], s.top, s.ids, s.saved, rows.view(K, -1)[:, V - 1: 2 * V - 1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K,V,n", [(5, 100, 300), (20000, 9, 4), (2, 300001, 700), (4000, 1031, 257)])
def test_more_entries_than_tokens_and_more_rows_than_blocks_at_once(K, V, n, dtype):
    rng = np.random.default_rng(V)
    draft = rng.normal(0, 2, (K, V)).astype(np.float32)
    ids = rng.integers(-1, V + 1, (K, n)).astype(np.int32)           # given several times, and places without an entry
    top = rng.normal(0, 2, (K, n)).astype(np.float32)
    s = Step(draft, top, ids, dtype)
    s.forward()
    some = np.unique(np.linspace(0, K - 1, 60).astype(int))
    at = torch.as_tensor(some, device=G.DEV)
    total, losses = float(s.total), s.loss.double().cpu().numpy()
    s.host, s.loss, s.top, s.ids = s.host[some], s.loss[at], s.top[at], s.ids[at]
    kept, whole = s.saved, s.total.clone()
    s.saved, s.total = s.saved[at], s.loss.double().sum().float()
    check_loss(s, TO.distill_loss(s.host, top[some], ids[some]))
    assert abs(total - losses.sum()) <= 2.0**-23 * losses.sum()
    s.saved, s.total, s.top, s.ids = kept, whole, dev(top), dev(ids, torch.int32)
    s.backward()
    got = s.grad[at].float().cpu().numpy()
    want = TO.distill_grad(s.host, top[some], ids[some], kept[at].cpu().numpy())
    # a token's weights, at most n of them that add up to 1: (n + 4) roundings of 32 bits; exponents of at most 64 rounded three times
    tol = (n + 4 + 3 * 64 + 8) * 2.0**-24 + (2.0**-8 if dtype == "bf16" else 0) * np.abs(want)
    assert (np.abs(got - want) <= tol).all(), np.abs(got - want).max()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_arrays_that_begin_at_any_number(dtype):
    """Hidden states, entries and losses 4 bytes behind a boundary of 16."""
    K, V, n, h = 9, 501, 33, 16
    _, draft, top, ids, feat, _ = make(25, K, V, n, h)
    s = Step(draft, top, ids, dtype, feat=feat, target_lse=np.full(K, 20.0, np.float32), seq=np.zeros(K), tau_seq=0.6)
    def shift(t):
        store = torch.zeros(t.numel() + 1, device=G.DEV, dtype=t.dtype)
        store[1:] = t.reshape(-1)
        return store[1:].view(t.shape)
    s.top, s.ids, s.loss, s.total = (shift(t) for t in (s.top, s.ids, s.loss, s.total))
    for name in ("feat", "target_lse", "seq"):
        s.kw[name] = shift(s.kw[name])
    s.forward()
    check_loss(s, TO.distill_loss(s.host, top, ids, target_lse=np.full(K, 20.0), feat=feat, seq=np.zeros(K), tau=0.6))
    s.backward(grad_loss=shift(torch.ones(K, device=G.DEV)))
    check_grad(s, s.saved.cpu().numpy(), np.ones(K), 1.0, dtype=dtype)
