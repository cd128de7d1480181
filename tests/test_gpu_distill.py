"""GPU parity of the loss on stored target logits and its gradient against their 64-bit restatements, within bounds that count
the roundings of 32-bit exponentials and sums."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as TO
from paper_2605_07230_b200 import binding as cb
from tests import gpu_util as G

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def dev(a, dtype=torch.float32):
    return None if a is None else torch.as_tensor(np.asarray(a), device=G.DEV).to(dtype)


def make(seed, K, V, n, h=8):
    """A target with a few likely codes, its n largest logits in no order, a noisy drafter, drifting hidden states."""
    rng = np.random.default_rng(seed)
    target = (rng.normal(0, 2.6, 256)[np.arange(V) % 256][None, :] + rng.normal(0, 0.3, (K, V))).astype(np.float32)
    draft = (target / 1.5 + rng.normal(0, 0.5, (K, V))).astype(np.float32)
    ids = np.argsort(-target, 1)[:, :n]
    ids = np.take_along_axis(ids, np.argsort(rng.random(ids.shape), 1), 1).astype(np.int32)
    feat = np.cumsum(rng.standard_normal((K, h)), 0).astype(np.float32)
    return target, draft, np.take_along_axis(target, ids, 1), ids, feat, rng


class Step:
    """Device arrays of one loss and its gradient; rows of logits `gap` elements apart, `lead` elements into their memory."""

    def __init__(self, draft, top, ids, dtype="f32", gap=0, lead=0, in_place=False, **kw):
        K, V = draft.shape
        store = torch.full((K * (V + gap) + lead + 8,), float("nan"), device=G.DEV, dtype=DT[dtype])
        self.draft = store[lead: lead + K * (V + gap)].view(K, V + gap)[:, :V]
        self.draft.copy_(dev(draft))
        self.host = self.draft.float().cpu().numpy()
        self.top, self.ids = dev(top), dev(ids, torch.int32)
        self.kw = {k: dev(v, torch.int32 if k == "seq" else torch.float32) if k in ("feat", "seq", "target_lse") else v for k, v in kw.items()}
        self.loss, self.saved, self.total = (torch.full(s, float("nan"), device=G.DEV) for s in ((K,), (K, 4), (1,)))
        self.grad_store = store if in_place else torch.full_like(store, float("nan"))
        self.grad = self.grad_store[lead: lead + K * (V + gap)].view(K, V + gap)[:, :V]

    def forward(self):
        cb.cascade_distill_loss(self.draft, self.top, self.ids, self.loss, self.saved, total=self.total, **self.kw)

    def backward(self, **kw):
        cb.cascade_distill_grad(self.draft, self.top, self.ids, self.saved, self.grad, temperature=self.kw.get("temperature", 1.0), **kw)


def spread(x, T):
    x = np.asarray(x, np.float64)
    x = x[np.isfinite(x)] / T
    return float(x.max() - x.min()) if x.size else 0.0


def sum_error(x, T, terms):
    """Relative error of a sum of exponentials: the exponential's own 2^-22, its argument (three roundings of at most the spread
    in units of ln 2, back by ln 2), and the additions of a thread, a warp, a block and a cluster."""
    return 2.0**-22 + 3 * spread(x, T) * 2.0**-24 + (terms / 128 + 40) * 2.0**-24


def check_loss(s, ref, T=1.0):
    loss, saved, cosine = ref
    K, V = s.host.shape
    got, kept = s.loss.cpu().numpy().astype(np.float64), s.saved.cpu().numpy().astype(np.float64)
    for k in range(K):
        w = saved[k, 3]
        if not np.isnan(cosine[k]) and abs(cosine[k] - s.kw.get("tau_seq", 0.5)) < 1e-12:
            continue
        assert kept[k, 3] == w, k
        e = sum_error(s.host[k], T, V) + sum_error(s.top[k].cpu().numpy(), T, s.ids.shape[1])
        # loss = w (Q log Z + sum q (m - d)): both parts are positive; log Z is off by e, the weights and products by e relatively
        assert abs(got[k] - loss[k]) <= w * e * (saved[k, 2] + 2 * abs(loss[k]) / max(w, 1)) + 2.0**-23 * abs(loss[k]), (k, got[k], loss[k])
        assert abs(kept[k, 0] - saved[k, 0]) <= e + 2.0**-23 * abs(saved[k, 0]) and abs(kept[k, 1] - saved[k, 1]) <= e + 2.0**-23 * abs(saved[k, 1])
        assert abs(kept[k, 2] - saved[k, 2]) <= (e + 3 * abs(saved[k, 1]) * 2.0**-24) * saved[k, 2] + 1e-30
    assert abs(float(s.total) - got.sum()) <= 2.0**-23 * np.abs(got).sum()


def check_grad(s, kept, up, scale, T=1.0, dtype="f32"):
    """Against the formula at the saved rows that the call itself read."""
    K, V = s.host.shape
    want = TO.distill_grad(s.host, s.top.cpu().numpy(), s.ids.cpu().numpy(), kept, up, scale, T)
    got = s.grad.float().cpu().numpy().astype(np.float64)
    half = 2.0**-8 if dtype == "bf16" else 2.0**-24
    for k in range(K):
        lse, t_lse, mass, w = (float(x) for x in kept[k])
        f = abs(w * (1 if up is None else float(up[k])) * scale / T)
        x = s.host[k].astype(np.float64) / T
        p = np.zeros(V) if f == 0 else mass * np.exp(x - lse)
        q = p - want[k] / (f or 1) * np.sign(w * (1 if up is None else float(up[k])) * scale)
        t = np.abs(s.top[k].cpu().numpy().astype(np.float64)[np.isfinite(s.top[k].cpu().numpy())]).max(initial=0) / T + abs(t_lse)
        with np.errstate(invalid="ignore"):
            e_p = 2.0**-22 + np.where(np.isfinite(x), np.abs(x) + 3 * np.abs(x - lse), 0.0) * 2.0**-23
        e_q = 2.0**-22 + 4 * t * 2.0**-23
        tol = f * (np.abs(p) * e_p + np.abs(q) * e_q) * (1 + half) + (half + 2.0**-22) * np.abs(want[k]) + 1e-37
        bad = np.abs(got[k] - want[k]) > tol
        assert not bad.any(), (k, np.flatnonzero(bad)[:4], got[k][bad][:4], want[k][bad][:4], tol[bad][:4])


SIZES = [(1, 1, 1), (3, 7, 2), (5, 129, 129), (2, 4097, 600), (16, 16384, 2000), (1, 65536, 3000), (5, 10007, 333), (500, 300, 17)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K,V,n", SIZES)
def test_loss_and_gradient(K, V, n, dtype):
    target, draft, top, ids, feat, rng = make(K + V, K, V, n)
    seq = np.sort(rng.integers(0, 2, K))
    seq[rng.random(K) < 0.1] = -1
    s = Step(draft, top, ids, dtype, feat=feat, seq=seq, tau_seq=0.3, c=2.0)
    s.forward()
    ref = TO.distill_loss(s.host, top, ids, feat=feat, seq=seq, tau=0.3, c=2.0)
    check_loss(s, ref)
    up = rng.normal(0, 1, K).astype(np.float32)
    s.backward(grad_loss=dev(up), scale=0.25)
    check_grad(s, s.saved.cpu().numpy(), up, 0.25, dtype=dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("temperature,given", [(0.5, False), (3.0, True), (1.0, True)])
def test_temperature_and_the_targets_own_sum(temperature, given, dtype):
    target, draft, top, ids, feat, rng = make(11, 9, 2001, 150)
    lse = np.log(np.exp(target.astype(np.float64) / temperature).sum(1)).astype(np.float32) if given else None
    s = Step(draft, top, ids, dtype, target_lse=lse, temperature=temperature)
    s.forward()
    check_loss(s, TO.distill_loss(s.host, top, ids, target_lse=lse, temperature=temperature), temperature)
    if given:
        assert (s.saved[:, 2] < 1).all()
    s.backward()
    check_grad(s, s.saved.cpu().numpy(), None, 1.0, temperature, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gap,lead", [(0, 1), (5, 0), (3, 3), (8, 4)])
@pytest.mark.parametrize("in_place", [False, True])
def test_rows_apart_at_any_element(dtype, gap, lead, in_place):
    K, V = 7, 1003
    _, draft, top, ids, _, _ = make(5, K, V, 40)
    s = Step(draft, top, ids, dtype, gap, lead, in_place)
    s.forward()
    check_loss(s, TO.distill_loss(s.host, top, ids))
    s.backward()
    check_grad(s, s.saved.cpu().numpy(), None, 1.0, dtype=dtype)
    rest = torch.ones_like(s.grad_store, dtype=torch.bool)           # nothing between the rows was written
    rest[lead: lead + K * (V + gap)].view(K, V + gap)[:, :V] = False
    assert s.grad_store[rest].isnan().all()


def test_gradient_rows_with_other_boundaries_than_the_logits():
    K, V = 6, 777
    _, draft, top, ids, _, _ = make(6, K, V, 30)
    s = Step(draft, top, ids, "bf16", gap=1)
    s.forward()
    store = torch.full((K, V + 4), float("nan"), device=G.DEV, dtype=torch.bfloat16)
    s.grad = store[:, 3: 3 + V]
    s.backward()
    check_grad(s, s.saved.cpu().numpy(), None, 1.0, dtype="bf16")
    assert store[:, :3].isnan().all() and store[:, 3 + V:].isnan().all()


def test_tokens_given_more_than_once_add_up_the_same_way_every_time():
    K, V, n = 40, 9000, 700
    _, draft, top, ids, _, rng = make(7, K, V, n)
    ids[:, 1:200] = ids[:, :1]                                       # one token two hundred times
    ids[3] = 8999
    s = Step(draft, top, ids)
    s.forward()
    check_loss(s, TO.distill_loss(s.host, top, ids))
    s.backward()
    kept = s.saved.cpu().numpy()
    want = TO.distill_grad(s.host, top, ids, kept)
    # up to n weights summed in 32 bits: (n + 4) roundings of a sum that is at most 1
    assert np.abs(s.grad.cpu().numpy() - want).max() <= (n + 60) * 2.0**-24
    first = s.grad.clone()
    for _ in range(5):
        s.backward()
        assert torch.equal(first, s.grad)


def test_places_without_an_entry_and_positions_without_any():
    K, V, n = 4, 500, 50
    _, draft, top, ids, _, _ = make(8, K, V, n)
    ids[0, ::3], ids[1], ids[2, 5] = -1, [-1, V] * (n // 2), 2**31 - 1
    top[3] = -np.inf
    top[0, 1] = -np.inf
    top[2, 5] = np.nan                                               # (not an entry: its logit is never used)
    s = Step(draft, top, ids)
    s.forward()
    check_loss(s, TO.distill_loss(s.host, top, ids))
    assert s.loss[1] == 0 and s.loss[3] == 0 and s.saved[1, 2] == 0 and s.saved[3, 2] == 0
    s.backward()
    check_grad(s, s.saved.cpu().numpy(), None, 1.0)
    assert not s.grad[1].any() and not s.grad[3].any()


@pytest.mark.parametrize("V", [600, 65536])
def test_infinities_and_values_that_are_no_numbers(V):
    K, n = 6, 20
    _, draft, top, ids, _, _ = make(9, K, V, n)
    ids, top = np.sort(ids, 1), np.take_along_axis(top, np.argsort(ids, 1), 1)
    out = np.setdiff1d(np.arange(V), ids.ravel())
    draft[0, out[:100]] = -np.inf                                    # weighs nothing, and nothing of the target lies there
    draft[1, ids[1, 0]] = -np.inf                                    # the target wants what the drafter excludes
    draft[2, out[3]] = np.nan
    draft[3, out[4]] = np.inf
    draft[4] = np.nan                                                # padding: whatever it holds
    top[5, 3] = np.nan
    seq = np.array([0, 0, 0, 0, -1, 0])
    s = Step(draft, top, ids, seq=seq)
    s.forward()
    loss = s.loss.cpu().numpy()
    ref = TO.distill_loss(s.host[:1], top[:1], ids[:1])
    assert abs(loss[0] - ref[0][0]) < 1e-4 * ref[0][0]
    assert loss[1] == np.inf and np.isnan(loss[[2, 3, 5]]).all() and loss[4] == 0
    s.backward()
    g = s.grad
    assert g[0].isfinite().all() and not g[0, torch.as_tensor(out[:100].copy(), device=G.DEV)].any()
    assert g[1].isfinite().all() and g[1, int(ids[1, 0])] < 0
    assert g[2].isnan().all() and g[3].isnan().all() and not g[4].any()
    assert g[5, int(ids[5, 3])].isnan()


def test_scale_of_zero_writes_zeros_whatever_the_logits_hold():
    _, draft, top, ids, _, _ = make(10, 3, 100, 5)
    draft[:] = np.nan
    s = Step(draft, top, ids)
    s.forward()
    s.backward(scale=0.0)
    assert not s.grad.any() and not s.grad.isnan().any()
    s.grad.fill_(7.0)
    s.backward(grad_loss=torch.zeros(3, device=G.DEV))
    assert not s.grad.any()


def test_recorded_and_replayed_on_another_stream():
    _, draft, top, ids, feat, _ = make(12, 12, 5000, 100)
    s = Step(draft, top, ids, feat=feat)
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        s.forward()
        s.backward()
    other = draft[::-1].copy()
    s.draft.copy_(dev(other))
    s.host = other
    graph.replay()
    torch.cuda.synchronize()
    check_loss(s, TO.distill_loss(other, top, ids, feat=feat))
    check_grad(s, s.saved.cpu().numpy(), None, 1.0)


def test_binding_checks_what_it_is_given():
    _, draft, top, ids, _, _ = make(13, 4, 64, 6)
    s = Step(draft, top, ids)
    for bad in (dict(draft=s.draft.half()), dict(draft=s.draft.t()), dict(top=s.top[:, :5]), dict(ids=s.ids.long()), dict(loss=s.loss[:3]),
                dict(saved=s.saved[:, :3]), dict(saved=s.saved.t().contiguous().t()), dict(draft=s.draft.cpu())):
        a = dict(draft=s.draft, top=s.top, ids=s.ids, loss=s.loss, saved=s.saved)
        a.update(bad)
        with pytest.raises(ValueError):
            cb.cascade_distill_loss(a["draft"], a["top"], a["ids"], a["loss"], a["saved"])
    with pytest.raises(ValueError):
        cb.cascade_distill_grad(s.draft, s.top, s.ids, s.saved, s.grad.bfloat16())
    with pytest.raises(cb.CascadeError):
        cb.cascade_distill_grad(s.draft, s.top, s.ids, s.saved, s.grad, temperature=0.0)
