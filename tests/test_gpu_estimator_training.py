"""The estimator's training path: its gradients against a 64-bit reverse pass of the same formulas, and what it trains as the
estimator that an engine predicts with."""
import numpy as np
import pytest
import torch

from oracle import moe_oracle as O
from paper_2603_19289_amd import workload as W
from tests.helpers import build, small_workload

pytestmark = pytest.mark.gpu

NAMES = ("proj", "layer_emb", "ffn_in", "ffn_out", "ln_gain", "ln_bias", "head")


def batch(wl, n, tokens, seed):
    g = torch.Generator().manual_seed(seed)
    signal = torch.randn(n, tokens, wl.hidden, generator=g)
    teacher = 1.5 * torch.randn(n, tokens, wl.n_experts, generator=g)
    ids = teacher.topk(wl.top_k, -1).indices.to(torch.int32)
    valid = torch.rand(n, tokens, generator=g) < 0.8
    return signal, teacher, ids, valid


def decoded(est):
    return {k: torch.from_numpy(O.decode_weights(v) if v.dtype == np.uint16 else v.astype(np.float64)) for k, v in est.items()}


def reverse_pass(est, layers, signal, teacher, ids, valid, coef):
    """Losses and gradients in 64 bits, by torch's differentiation of elementary operations."""
    w = {k: v.clone().requires_grad_() for k, v in decoded(est).items()}
    n, tokens, _ = signal.shape
    u = signal.double() @ w["proj"].T + w["layer_emb"][list(layers)][:, None]
    h = u @ w["ffn_in"].T
    v = u + (h * torch.sigmoid(h)) @ w["ffn_out"].T
    c = v - v.mean(-1, keepdim=True)
    y = c / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-5) * w["ln_gain"] + w["ln_bias"]
    z = y @ w["head"].T
    live = valid.double()
    p, log_q = torch.softmax(teacher.double(), -1), z - torch.logsumexp(z, -1, keepdim=True)
    loss = ((p * (p.log() - log_q)).sum(-1) * live).sum() / live.sum()
    counts = torch.bincount(ids[valid].reshape(-1).long(), minlength=z.shape[-1])
    f = counts.double() / live.sum() / ids.shape[-1]
    balance = coef * z.shape[-1] * (f * (log_q.exp() * live[..., None]).sum((0, 1)) / live.sum()).sum()
    (loss + balance).backward()
    return loss.item(), balance.item(), counts, {k: t.grad for k, t in w.items()}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_equal_those_of_a_64_bit_reverse_pass(dtype):
    """Relative to the largest gradient of a table.  float32: six products of at most 264 terms one after the other, each off by at
    most 264 u of its terms' magnitudes, which are below 20 times what they add up to here: 6 * 264 * 20 * 2^-24 = 2e-3.  bfloat16: ten
    roundings of 2^-8 on the way to any gradient, not all of one sign: their sum, 4e-2."""
    from paper_2603_19289_amd import training as T
    wl = small_workload(name="training", n_layers=5, hidden=264, n_experts=12, top_k=3, inter=200, dtype=dtype, batch=1, tokens=1, slots=6, seed=5)
    est = W.make_estimator(wl, m=3, n=2)
    layers = [3, 0, 2]
    signal, teacher, ids, valid = batch(wl, 3, 37, 1)
    trainer = T.EstimatorTrainer(est, balance_coef=0.1)
    out, grads = trainer.gradients(layers, signal.cuda(), teacher.cuda(), ids.cuda(), valid.cuda())
    loss, balance, counts, want = reverse_pass(est, layers, signal, teacher, ids, valid, 0.1)
    tol = 2e-3 if dtype == "f32" else 4e-2
    assert abs(out["loss"].item() - loss) < tol * loss and abs(out["balance"].item() - balance) < tol * balance
    assert torch.equal(out["counts"].cpu().long(), counts)
    for k in NAMES:
        off = (grads[k].cpu().double() - want[k]).abs().max() / want[k].abs().max()
        assert off < tol, (k, off)
    assert not grads["layer_emb"][[1, 4]].any()
    for bad in ([0, 0, 1], [0, 1], [0, 1, 5], [0, 1, -1]):                   # refused before anything is looked up
        with pytest.raises(ValueError):
            trainer.gradients(bad, signal.cuda(), teacher.cuda(), ids.cuda(), valid.cuda())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("state", ["f32", "f8"])
def test_an_engine_predicts_with_what_is_trained_in_its_memory(dtype, state):
    """The engine's own tables are trained in place between decode steps; its predictions are the oracle's with the trained tables."""
    from paper_2603_19289_amd import training as T
    from paper_2603_19289_amd.engine import engine_for
    wl = small_workload(name="training", n_layers=4, hidden=264, n_experts=12, top_k=3, inter=200, dtype=dtype, batch=3, tokens=1, slots=9, seed=6)
    res, ex, model = build(wl, "random")
    est = W.make_estimator(wl, m=3, n=2)
    eng = engine_for(wl, O.MODE_SPECULATIVE, res, ex, estimator=est)
    try:
        trainer = T.EstimatorTrainer(eng.est, lr=0.02, state=state, seed=1)
        for step in range(3):
            signal, teacher, ids, valid = (t.cuda() for t in batch(wl, 2, 50, 10 + step))
            trainer.step([step, 3], signal, teacher, ids, valid)
        torch.cuda.synchronize()
        trained = trainer.numpy_weights()
        for k in NAMES:
            now = eng.est[k].view(torch.int16).cpu().numpy().view(np.uint16) if eng.est[k].dtype == torch.bfloat16 else eng.est[k].cpu().numpy()
            assert np.array_equal(now, trained[k]) and not np.array_equal(trained[k], est[k]), k
        x0, eps = W.make_inputs(wl)
        advance = lambda t, l, r, o: W.advance_residual(wl, r, o, eps[t, l])  # noqa: E731
        trace = {}
        for name, weights in (("trained", trained), ("before", est)):
            orc = O.MoEOracle(model, O.MODE_SPECULATIVE, wl.slots, estimator=O.Estimator(**weights), estimator_layers=range(wl.n_layers))
            trace[name] = O.run_tokens(orc, x0, advance)
        eng.begin_token()
        for l in range(wl.n_layers):
            r, want = trace["trained"][0][l]
            _, got = eng.layer_step(l, torch.from_numpy(r.astype(np.float32)).cuda(), want_ids=True)
            torch.cuda.synchronize()
            assert np.array_equal(got["exec_ids"].cpu().numpy(), want.exec_ids), l
            if l + 1 < wl.n_layers:
                assert np.array_equal(got["next_ids"].cpu().numpy(), trace["trained"][0][l + 1][1].exec_ids), l
        first = trace["before"][0][1][1].exec_ids
        assert not np.array_equal(first, trace["trained"][0][1][1].exec_ids)     # training did change what is predicted
    finally:
        eng.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_padding_counts_for_nothing_whatever_it_holds(dtype):
    """NaN, infinities and the type's largest values in the signal and the logits of rows that do not count: the bits of zeros there,
    in the losses, in every gradient and in the tables after a step."""
    from paper_2603_19289_amd import training as T
    wl = small_workload(name="training", n_layers=5, hidden=264, n_experts=12, top_k=3, inter=200, dtype=dtype, batch=1, tokens=1, slots=6, seed=5)
    est = W.make_estimator(wl, m=3, n=2)
    signal, teacher, ids, valid = (t.cuda() for t in batch(wl, 3, 37, 1))
    valid[1] = False                                      # a layer of padding only
    want = None
    for junk in (0.0, float("nan"), float("inf"), -float("inf"), torch.finfo(torch.float32).max):
        trainer = T.EstimatorTrainer(est, balance_coef=0.1, state="f8")
        fill = lambda t: torch.where(valid[..., None], t, torch.full_like(t, junk))  # noqa: E731
        for mask in (valid, valid.to(torch.uint8)):
            out, grads = trainer.gradients([3, 0, 2], fill(signal), fill(teacher), ids, mask)
            now = [*out.values(), *(grads[k] for k in NAMES)]
            want = want or now
            assert all(torch.isfinite(t).all() for t in now), junk
            assert all(torch.equal(a, b) for a, b in zip(now, want)), junk
        trainer.step([3, 0, 2], fill(signal), fill(teacher), ids, valid)
        assert all(torch.isfinite(t).all() for t in trainer.weights.values()), junk
    for bad in (valid[:2], valid.float(), valid[..., None]):
        with pytest.raises(ValueError):
            trainer.gradients([3, 0, 2], signal, teacher, ids, bad)


def test_a_balance_term_without_choices_is_refused():
    from paper_2603_19289_amd import training as T
    wl = small_workload(name="training", n_layers=5, hidden=264, n_experts=12, top_k=3, inter=200, dtype="f32", batch=1, tokens=1, slots=6, seed=5)
    signal, teacher, _, valid = (t.cuda() for t in batch(wl, 3, 37, 1))
    trainer = T.EstimatorTrainer(W.make_estimator(wl, m=3, n=2), balance_coef=0.1)
    before = {k: t.clone() for k, t in trainer.weights.items()}
    for call in (trainer.gradients, trainer.step):
        with pytest.raises(ValueError):
            call([3, 0, 2], signal, teacher, None, valid)
    assert all(torch.equal(before[k], t) for k, t in trainer.weights.items())
    trainer.balance_coef = 0.0
    assert "balance" not in trainer.step([3, 0, 2], signal, teacher, None, valid)


def logits_of(est, layers, signal):
    """The estimator's logits in 64 bits."""
    w = decoded(est)
    u = signal.double() @ w["proj"].T + w["layer_emb"][list(layers)][:, None]
    h = u @ w["ffn_in"].T
    v = u + (h * torch.sigmoid(h)) @ w["ffn_out"].T
    c = v - v.mean(-1, keepdim=True)
    return (c / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-5) * w["ln_gain"] + w["ln_bias"]) @ w["head"].T


def collapsed(est):
    """Weights that give expert 0 the largest logit whatever the signal: its row of the head lies along the bias that all outputs share."""
    bias = 0.4 * np.random.default_rng(3).standard_normal(len(est["ln_bias"])).astype(np.float32)
    head = est["head"].copy()
    head[0] = 0.3 * bias
    return {**est, "ln_gain": 0.05 * est["ln_gain"], "ln_bias": bias, "head": head}


@pytest.mark.parametrize("fallen", [False, True])
def test_the_balance_term_is_of_the_estimators_own_choices(fallen):
    """Under balanced routers: f of the top-k of the estimator's logits in the loss, the counts and every gradient, by the 64-bit
    reverse pass with those choices.  No row's choice hangs on rounding: four products of at most 264 terms move z by at most 4 * 264 *
    2^-24 of their terms' magnitudes, which are below 5 times the largest logit: 3e-4 of that."""
    from paper_2603_19289_amd import training as T
    wl = small_workload(name="training", n_layers=5, hidden=264, n_experts=12, top_k=3, inter=200, dtype="f32", batch=1, tokens=1, slots=6, seed=5)
    est = W.make_estimator(wl, m=3, n=2)
    est = collapsed(est) if fallen else est
    layers = [3, 0, 2]
    signal, teacher, _, valid = batch(wl, 3, 37, 1)
    teacher[:] = 0.0
    z = logits_of(est, layers, signal)
    ranked, chosen = z.sort(-1, descending=True)
    assert (ranked[..., 2] - ranked[..., 3]).min() > 3e-4 * z.abs().max()      # in 64 bits, before anything runs
    trainer = T.EstimatorTrainer(est, balance_coef=0.1, top_k=3)
    out, grads = trainer.gradients(layers, signal.cuda(), teacher.cuda(), valid=valid.cuda())
    loss, balance, counts, want = reverse_pass(est, layers, signal, teacher, chosen[..., :3], valid, 0.1)
    assert torch.equal(out["counts"].cpu().long(), counts) and (not fallen or counts[0] == valid.sum())
    assert abs(out["loss"].item() - loss) < 2e-3 * loss and abs(out["balance"].item() - balance) < 2e-3 * balance
    for k in NAMES:
        assert (grads[k].cpu().double() - want[k]).abs().max() < 2e-3 * want[k].abs().max(), k
    without = T.EstimatorTrainer(est, top_k=3).gradients(layers, signal.cuda(), teacher.cuda(), valid=valid.cuda())
    assert torch.equal(without[0]["counts"], out["counts"])
    if fallen:                                             # it is pushed: by more than rounding, in the head's row of expert 0
        assert (grads["head"][0] - without[1]["head"][0]).abs().max() > 0.01 * without[1]["head"].abs().max()
    for bad in (0, 13):
        with pytest.raises(ValueError):
            T.EstimatorTrainer(est, top_k=bad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("state", ["f32", "f8"])
def test_training_that_is_resumed_goes_on_as_if_it_had_not_stopped(dtype, state):
    """Masters, moments and the step's number through host memory into a new trainer: the bits of the one that went on."""
    from paper_2603_19289_amd import training as T
    wl = small_workload(name="training", n_layers=5, hidden=264, n_experts=12, top_k=3, inter=200, dtype=dtype, batch=1, tokens=1, slots=6, seed=5)
    est = W.make_estimator(wl, m=3, n=2)
    steps = [tuple(t.cuda() for t in batch(wl, 3, 37, s)) for s in range(4)]
    whole = T.EstimatorTrainer(est, lr=1e-3, state=state, seed=4)
    for signal, teacher, _, valid in steps[:2]:
        whole.step([3, 0, 2], signal, teacher, valid=valid)
    saved = {k: t.cpu().clone() for k, t in whole.masters().items()}
    moments = {k: [t.cpu().clone() for t in ts] for k, ts in whole.optimizer.states().items()}
    weights, number = whole.numpy_weights(), whole.optimizer.steps
    for signal, teacher, _, valid in steps[2:]:
        whole.step([3, 0, 2], signal, teacher, valid=valid)
    resumed = T.EstimatorTrainer(weights, lr=1e-3, state=state, seed=4, masters={k: t.cuda() for k, t in saved.items()},
                                 states={k: [t.cuda() for t in ts] for k, ts in moments.items()}, steps=number)
    assert all(np.array_equal(weights[k], v) for k, v in resumed.numpy_weights().items())
    for signal, teacher, _, valid in steps[2:]:
        resumed.step([3, 0, 2], signal, teacher, valid=valid)
    for a, b in ((whole.masters(), resumed.masters()), (whole.weights, resumed.weights)):
        assert all(torch.equal(a[k], b[k]) for k in NAMES)
    for k, ts in whole.optimizer.states().items():
        assert all(torch.equal(a, b) for a, b in zip(ts, resumed.optimizer.states()[k]))
    with pytest.raises(ValueError):
        T.EstimatorTrainer(est, masters={**{k: t.cuda() for k, t in saved.items()}, "head": saved["head"][:, 1:].cuda()})
    with pytest.raises(ValueError):
        T.EstimatorTrainer(est, masters={k: t.cuda().to(torch.float16) for k, t in saved.items()})


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,tokens", [(3, 0), (0, 5), (1, 1)])
def test_batches_of_nothing_and_of_one_token(n, tokens, dtype):
    """Without rows: losses, counts and gradients of zero; one row: finite ones."""
    from paper_2603_19289_amd import training as T
    wl = small_workload(name="training", n_layers=5, hidden=264, n_experts=12, top_k=3, inter=200, dtype=dtype, batch=1, tokens=1, slots=6, seed=5)
    signal, teacher, _, valid = (t.cuda() for t in batch(wl, n, tokens, 1))
    trainer = T.EstimatorTrainer(W.make_estimator(wl, m=3, n=2), balance_coef=0.1, top_k=3)
    for mask in (None, valid):
        out, grads = trainer.gradients(range(n), signal, teacher, valid=mask)
        assert all(grads[k].shape == trainer.weights[k].shape and torch.isfinite(grads[k]).all() for k in NAMES)
        if n * tokens == 0:
            assert out["loss"].item() == out["balance"].item() == 0.0 and not out["counts"].any()
            assert not any(g.any() for g in grads.values())
    trainer.step(range(n), signal, teacher, valid=valid)
    assert all(torch.isfinite(t).all() for t in trainer.weights.values())


def test_layers_named_by_a_tensor():
    """As by a list; the same one twice is refused, as only one of its gradients would be kept."""
    from paper_2603_19289_amd import training as T
    wl = small_workload(name="training", n_layers=5, hidden=264, n_experts=12, top_k=3, inter=200, dtype="f32", batch=1, tokens=1, slots=6, seed=5)
    signal, teacher, _, valid = (t.cuda() for t in batch(wl, 2, 9, 1))
    trainer = T.EstimatorTrainer(W.make_estimator(wl, m=3, n=2))
    want = trainer.gradients([3, 0], signal, teacher, valid=valid)[1]
    for layers in (torch.tensor([3, 0]), torch.tensor([3, 0], device="cuda"), np.array([3, 0])):
        got = trainer.gradients(layers, signal, teacher, valid=valid)[1]
        assert all(torch.equal(got[k], want[k]) for k in NAMES)
        with pytest.raises(ValueError):
            trainer.gradients(layers * 0, signal, teacher, valid=valid)
    with pytest.raises(TypeError):
        trainer.gradients([0.5, 1.5], signal, teacher, valid=valid)
