"""Which masks the layers of a residual block draw (no GPU: the mask's definition in the kernel's place)."""
import copy

import pytest
import torch
from torch.utils.checkpoint import checkpoint

from paper_2310_03675_amd import autograd as A
from residual_block import dropped, kept


@pytest.fixture
def on_the_host(monkeypatch):
    def dropout(x, d, residual=None):
        y = dropped(x, d).to(x.dtype)
        return y if residual is None else residual + y

    monkeypatch.setattr(A.B, "dropout", dropout)


@pytest.mark.parametrize("reentrant", [True, False])
def test_a_forward_pass_made_again_has_its_masks(on_the_host, reentrant):
    """Two layers, one of them called twice, in segments that the backward pass makes again in the other order: the gradient goes through
    the output's masks."""
    one, two = A.ResidualDropout(0.5, seed=1, layer_id=1), A.ResidualDropout(0.3, seed=1, layer_id=2)
    first, second = (lambda v: two(one(v))), (lambda v: one(v))
    for step in range(3):
        x = torch.ones(400, requires_grad=True)
        y = checkpoint(second, checkpoint(first, x, use_reentrant=reentrant), use_reentrant=reentrant)
        y.sum().backward()
        assert torch.equal(x.grad, y.detach())                  # (linear in x, which is one)
        masks = [kept(400, p, 1 + s, i) for p, s, i in ((0.5, 2 * step, 1), (0.3, step, 2), (0.5, 2 * step + 1, 1))]
        assert torch.equal(y != 0, masks[0] & masks[1] & masks[2])
    assert one.masks.step == 6 and two.masks.step == 3


def test_several_passes_before_their_backward_passes(on_the_host):
    m = A.ResidualDropout(0.5, seed=4)
    xs = [torch.ones(300, requires_grad=True) for _ in range(5)]
    ys = [checkpoint(m, x, use_reentrant=True) for x in xs]
    for x, y in list(zip(xs, ys))[::-1]:
        y.sum().backward()
        assert torch.equal(x.grad, y.detach())
    assert len({tuple(y.tolist()) for y in ys}) == 5


def test_a_forward_pass_that_cannot_be_told_is_refused(on_the_host):
    m = A.ResidualDropout(0.5)
    x = torch.ones(100, requires_grad=True)
    y = checkpoint(m, x, use_reentrant=True, preserve_rng_state=False)
    with pytest.raises(RuntimeError, match="random state"):
        y.sum().backward()


def test_a_counters_pass_made_again(on_the_host):
    m = A.ResidualDropout(0.5, seed=2)
    m.masks.counter = torch.zeros(1, dtype=torch.int64)
    state = torch.get_rng_state()
    for _ in range(2):
        x = torch.ones(300, requires_grad=True)
        y = checkpoint(m, x, use_reentrant=True, preserve_rng_state=False)
        y.sum().backward()
        assert torch.equal(x.grad, y.detach())
        m.masks.counter.add_(1)
    assert torch.equal(torch.get_rng_state(), state)


def test_how_many_calls_are_kept():
    m = A.ResidualDropout(0.5).masks
    for k in range(m.REMEMBERED + 10):
        assert m.next(True).seed == k
    assert len(m._drawn) == m.REMEMBERED
    m.step = 5
    assert m.next(True).seed == 5 and len(m._drawn) == 1


def test_layers_without_an_id_have_masks_of_their_own(on_the_host):
    layers = [A.ResidualDropout(0.5) for _ in range(4)]
    layers += [copy.deepcopy(layers[0]), copy.deepcopy(torch.nn.Sequential(layers[0]))[0]]
    ys = [m(torch.ones(400)) for m in layers]
    for i, y in enumerate(ys):
        for z in ys[:i]:
            assert 0.35 < float(((y != 0) == (z != 0)).double().mean()) < 0.65         # (half; six standard deviations of 400 draws)
    ids = [m.masks.layer_id for m in layers + [A.ResidualNorm(8, p=0.1), A.ResidualNorm(8)]]
    assert len(set(ids)) == 8 and all(2 ** 31 <= i < 2 ** 32 for i in ids)
    # one that has an id keeps it
    m = A.ResidualDropout(0.5, layer_id=3)
    assert m.masks.layer_id == 3 and copy.deepcopy(m).masks.layer_id == 3
    m.masks.counter = torch.zeros(1, dtype=torch.int64)
    assert torch.equal(m(torch.ones(400)), copy.deepcopy(m)(torch.ones(400)))


def test_a_run_that_is_taken_up_again_goes_on_with_its_masks(on_the_host, tmp_path):
    new = lambda: torch.nn.Sequential(A.ResidualDropout(0.5, seed=7, layer_id=1), A.ResidualDropout(0.2, layer_id=2))
    x, net, again = torch.ones(300), new(), new()
    for _ in range(3):
        net(x)
    torch.save(net.state_dict(), tmp_path / "state")
    want = [net(x) for _ in range(2)]
    held = torch.load(tmp_path / "state", weights_only=True)
    again.load_state_dict(held)
    assert list(held) == ["0.step", "1.step"] and all(torch.equal(again(x), y) for y in want)
    again.load_state_dict(held)                                 # (it is not used up)
    assert torch.equal(again(x), want[0])


def test_states_of_layers_with_and_without_dropout():
    norm, plain = A.ResidualNorm(8, p=0.1), A.ResidualNorm(8)
    assert list(norm.state_dict()) == ["weight", "bias", "step"] and list(plain.state_dict()) == ["weight", "bias"]
    norm.masks.step = 9
    norm.load_state_dict(plain.state_dict())                    # one from before has no step
    assert norm.masks.step == 9
    plain.load_state_dict(norm.state_dict())
    with pytest.raises(RuntimeError, match="bias"):
        norm.load_state_dict({"weight": torch.ones(8), "step": torch.tensor(2)})
    with pytest.raises(RuntimeError, match="other"):
        norm.load_state_dict({**norm.state_dict(), "other": torch.ones(8)})


def test_a_description_that_changes_before_the_backward_pass(on_the_host, monkeypatch):
    """One object for two calls, with another id for the second."""
    how, x = A.B.Dropout(0.5, seed=1, tensor_id=1), torch.ones(300, requires_grad=True)
    y = A.Dropout.apply(x, None, how)
    how.tensor_id, how.seed, how.p = 2, 5, 0.1
    y.sum().backward()
    assert torch.equal(x.grad, y.detach())

    seen = []
    monkeypatch.setattr(A.B, "layernorm_fwd", lambda x, w, b, eps, r, d: (x * 1, x * 1, torch.zeros(x.shape[:-1] + (2,))))
    monkeypatch.setattr(A.B, "layernorm_bwd", lambda dy, s, saved, w, ds, d, need: (seen.append((d.p, d.seed, d.tensor_id)), (dy, None, None, None))[1])
    y, _ = A.LayerNorm.apply(x.reshape(3, 100), None, None, None, 1e-5, how)
    how.tensor_id = 3
    y.sum().backward()
    assert seen == [(0.1, 5, 2)]
