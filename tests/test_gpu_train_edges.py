"""The differentiable policy loss where the caller's arrays change, have other shapes, or are differentiated twice."""
import pytest
import torch

from paper_2407_08103_b200 import cstr
from paper_2407_08103_b200.train import constrained_policy_loss
from synth.configs import config_dfas, config_vocab

from gpu_common import gpu_tables

DEV = "cuda:0"
pytestmark = pytest.mark.gpu


def batch(N=24, seed=3):
    """Two tables over one vocabulary, and the arguments of a loss over N rows."""
    vb, vo = config_vocab("api_1k")
    tables = gpu_tables([config_dfas("api_1k")[0]] * 2, vb, vo)
    g = torch.Generator(device=DEV).manual_seed(seed)
    logits = torch.randn(N, vo.size - 1, generator=g, device=DEV)

    def ints(n):
        return torch.randint(0, n, (N,), generator=g, device=DEV, dtype=torch.int32)

    def normal():
        return torch.randn(N, generator=g, device=DEV)
    from oracle import token_table
    d = config_dfas("api_1k")[0]
    allowed = torch.from_numpy(token_table(d[0], d[1], vb, vo)[0] >= 0).to(DEV)
    states = ints(allowed.shape[0])
    actions = (allowed[states.long()].float() + 1e-9).multinomial(1, generator=g)[:, 0].int()
    return dict(logits=logits, actions=actions, old_logp=normal() - 3.0, advantages=normal(), tables=tables,
                states=states, ref_logp=normal() - 3.0, weight=torch.rand(N, generator=g, device=DEV),
                row_table=ints(2), kl_coef=0.1)


def gradient(a, between=None, up=None):
    x = a["logits"].clone().requires_grad_()
    loss, _ = constrained_policy_loss(**dict(a, logits=x))
    if between:
        between()
    loss.backward(torch.ones_like(loss) if up is None else up)
    return x.grad


@pytest.mark.parametrize("name", ["states", "row_table", "actions", "old_logp", "advantages", "ref_logp", "weight"])
def test_the_gradient_is_that_of_the_arrays_as_they_were(name):
    a = batch()
    want = gradient(a)
    assert want.abs().sum() > 0
    # as a kernel writes them: autograd does not see it
    other = torch.full_like(a[name], -1)
    got = gradient(a, lambda: a[name].data.copy_(other))
    assert torch.equal(got, want)


def test_logits_without_gradient():
    a = batch()
    w = a["weight"].clone().requires_grad_()
    loss, _ = constrained_policy_loss(**dict(a, weight=w))
    assert torch.equal(loss.detach(), constrained_policy_loss(**a)[0])
    loss.sum().backward()                                  # differentiable in the logits only
    assert w.grad is None


def test_a_table_built_again_before_the_backward_pass_is_refused():
    vb, vo = config_vocab("api_1k")
    dfa = config_dfas("api_1k")[0]
    vocab, d = cstr.cstr_load_vocab(vb, vo), cstr.cstr_load_dfa(*dfa)
    table = cstr.cstr_table_create(vocab, dfa[0].shape[0])
    cstr.cstr_table_build(table, d)
    a = dict(batch(), tables=[table], row_table=None)
    assert torch.equal(gradient(a), gradient(dict(a, tables=table)))
    for again in (cstr.cstr_table_build, cstr.cstr_table_build_dense):
        with pytest.raises(RuntimeError, match="built again"):
            gradient(a, lambda: again(table, d))
    gradient(a)                                            # a loss taken after that is fine


def test_second_derivatives_are_refused():
    a = batch()
    x = a["logits"].clone().requires_grad_()
    loss, _ = constrained_policy_loss(**dict(a, logits=x))
    (g,) = torch.autograd.grad(loss.sum(), x, create_graph=True)
    assert torch.equal(g, gradient(a))
    with pytest.raises(RuntimeError, match="once only"):
        (g * x).sum().backward()                           # (the term through g must not be left out)


@pytest.mark.parametrize("name", ["weight", "states", "actions", "old_logp", "advantages", "ref_logp", "row_table"])
def test_per_row_arrays_of_other_shapes(name):
    # one entry per row is what counts: a column, or an array with entries to spare
    a = batch()
    want, up = gradient(a), torch.rand(24, device=DEV)
    want_up = gradient(a, up=up)
    for other in (a[name][:, None], torch.cat([a[name], a[name]])):
        assert torch.equal(gradient(dict(a, **{name: other})), want)
        assert torch.equal(gradient(dict(a, **{name: other}), up=up), want_up)
