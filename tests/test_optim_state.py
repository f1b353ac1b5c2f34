"""optim.AdamW and optim.MALT: copied, pickled, saved and loaded, without a GPU.  The kernel is stood in for."""
import copy
import pickle

import pytest
import torch


@pytest.fixture()
def steps(monkeypatch):
    """ops.adamw_step and adamw_state stood in for: the calls' keywords are kept."""
    from paper_2608_05088_amd import ops
    calls = []
    monkeypatch.setattr(ops, "adamw_state", lambda p, bits=32: torch.zeros((2, p.numel())) if bits == 32 else
                        torch.zeros(-(-p.numel() // 256) * 520, dtype=torch.uint8))

    def step(params, grads, states, **kw):
        calls.append(kw)
        for p, st in zip(params, states):
            p.sub_(kw["lr"])
            st.add_(1)

    monkeypatch.setattr(ops, "adamw_step", step)
    return calls


def adamw(sizes=(10, 5000), **kw):
    from paper_2608_05088_amd.optim import AdamW
    ps = [torch.nn.Parameter(torch.zeros(n)) for n in sizes]
    for p in ps:
        p.grad = torch.ones_like(p)
    return AdamW(ps, **kw), ps


@pytest.mark.parametrize("how", [copy.deepcopy, lambda x: pickle.loads(pickle.dumps(x))])
@pytest.mark.parametrize("stepped", [False, True])
def test_a_copy_steps_as_the_original(steps, how, stepped):
    opt, ps = adamw(bits=8, min_8bit=64, seed=11)
    if stepped:
        opt.step()
    other = how(opt)
    qs = [p for g in other.param_groups for p in g["params"]]
    assert (other.bits, other.min_8bit, other.seed) == (8, 64, 11)
    for q in qs:   # a pickled parameter keeps no gradient
        q.grad = torch.ones_like(q)
    steps.clear()
    opt.step(), other.step()
    assert steps[0] == steps[1] and steps[0]["seed"] >> 32 == 11
    for p, q in zip(ps, qs):
        assert p is not q and torch.equal(p, q) and other.state[q]["step"] == 1 + stepped
        assert opt.state[p]["moments"].dtype == other.state[q]["moments"].dtype == (torch.uint8 if p.numel() >= 64 else torch.float32)
        assert torch.equal(opt.state[p]["moments"], other.state[q]["moments"])
