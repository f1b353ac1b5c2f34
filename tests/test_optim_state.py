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


# ------------------------------------------------------------------- loading
def _torch_adamw(sizes=(10, 5000)):
    ps = [torch.nn.Parameter(torch.zeros(n)) for n in sizes]
    opt = torch.optim.AdamW(ps, lr=0.125)
    for p in ps:
        p.grad = torch.ones_like(p)
    opt.step()
    return opt


def _snapshot(opt, ps):
    return [(dict(opt.state[p]), {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in opt.state[p].items()}) for p in ps], \
           [{k: v for k, v in g.items() if k != "params"} for g in opt.param_groups]


def _unchanged(opt, ps, before):
    states, groups = before
    assert [{k: v for k, v in g.items() if k != "params"} for g in opt.param_groups] == groups
    for p, (same, values) in zip(ps, states):
        assert opt.state[p].keys() == same.keys()
        for k, v in opt.state[p].items():
            assert v is same[k] and (torch.equal(v, values[k]) if isinstance(v, torch.Tensor) else v == values[k])


@pytest.mark.parametrize("what", ["torch", "size", "bytes", "type", "count", "step", "no tensor", "part", "groups"])
def test_a_state_that_does_not_fit_is_refused_as_a_whole(steps, what):
    opt, ps = adamw(bits=8)
    opt.step()
    saved = copy.deepcopy(opt.state_dict())
    saved["param_groups"][0]["lr"] = 0.75
    st = saved["state"]
    if what == "torch":
        saved = _torch_adamw().state_dict()
    elif what == "size":
        st[0]["moments"] = torch.zeros(2, 11)
    elif what == "bytes":
        st[1]["moments"] = st[1]["moments"][:-1]
    elif what == "type":
        st[0]["moments"] = st[0]["moments"].bfloat16()
    elif what == "count":
        st[1]["step"] = -1
    elif what == "step":
        st[1]["step"] = None
    elif what == "no tensor":
        st[1]["moments"] = [0.0] * 10000
    elif what == "part":
        del st[1]["moments"]
    else:
        saved["param_groups"].append(dict(saved["param_groups"][0], params=[2]))
    before = _snapshot(opt, ps)
    with pytest.raises(ValueError):
        opt.load_state_dict(saved)
    _unchanged(opt, ps, before)
    opt.step()
    assert [opt.state[p]["step"] for p in ps] == [2, 2]


def test_parameters_that_have_not_stepped_are_saved_and_loaded(steps):
    opt, ps = adamw()
    ps[0].grad = None
    opt.step()
    other, qs = adamw()
    other.load_state_dict(opt.state_dict())
    assert not other.state[qs[0]] and other.state[qs[1]]["step"] == 1
    other.step()
    assert [other.state[q]["step"] for q in qs] == [1, 2]


def _malt(bits):
    from paper_2608_05088_amd.optim import MALT
    w, b, c = (torch.nn.Parameter(torch.zeros(s)) for s in ((8, 16), (16,), (5000,)))
    b.grad, c.grad = torch.ones(16), torch.ones(5000)
    opt = MALT([w, b, c], adamw_bits=bits, lr=0.5, adamw_lr=0.25)
    opt._adam.step()
    opt._resume[0] = {"state": torch.arange(10.0), "t": 3, "shapes": [(8, 16)], "variant": "malt"}
    return opt, (b, c)


@pytest.mark.parametrize("bits,other", [(None, 8), (None, 32), (8, None), (32, None)])
def test_the_other_adamws_state_is_refused_before_anything_changes(steps, bits, other):
    """A checkpoint of MALT with torch's AdamW in one with this module's, and the reverse."""
    opt, ps = _malt(other)
    saved, _ = _malt(bits)
    saved.param_groups[0]["lr"] = 0.75
    saved._resume[0] = dict(saved._resume[0], t=9)
    sd, before, plan = saved.state_dict(), _snapshot(opt._adam, ps), opt._resume[0]
    with pytest.raises(ValueError, match="AdamW"):
        opt.load_state_dict(sd)
    assert opt._resume[0] is plan and opt.param_groups[0]["lr"] == 0.5
    _unchanged(opt._adam, ps, before)
    for like in (None, 8):   # each its own kind
        a, pa = _malt(like)
        b, pb = _malt(like)
        a._adam.step()
        a._resume[0] = dict(a._resume[0], t=7)
        b.load_state_dict(a.state_dict())
        assert b._resume[0]["t"] == 7 and int(b._adam.state[pb[0]]["step"]) == 2


def test_a_later_group_that_does_not_fit_leaves_the_earlier_ones():
    """All of a state's shapes are looked at before the first group's is taken over."""
    from paper_2608_05088_amd.optim import MALT
    def two(n):
        opt = MALT([dict(params=[torch.nn.Parameter(torch.zeros(8, 16))]), dict(params=[torch.nn.Parameter(torch.zeros(4, n))])])
        opt._resume = [{"state": torch.zeros(1), "t": n, "shapes": [s], "variant": "malt"} for s in ((8, 16), (4, n))]
        return opt
    opt, other = two(8), two(16)
    before = list(opt._resume)
    with pytest.raises(ValueError, match="group 1"):
        opt.load_state_dict(other.state_dict())
    assert all(a is b for a, b in zip(opt._resume, before))


@pytest.mark.parametrize("own", [0, 7])
def test_a_resumed_run_rounds_as_the_first(steps, own, tmp_path):
    """The seed is part of what is saved; a state without one leaves the optimizer's own."""
    opt, ps = adamw(bits=8, seed=7)
    opt.step()
    torch.save(opt.state_dict(), tmp_path / "o.pt")
    saved = torch.load(tmp_path / "o.pt", weights_only=True)
    other, qs = adamw(bits=8, seed=own)
    other.load_state_dict(saved)
    steps.clear()
    opt.step(), other.step()
    assert steps[0] == steps[1] and steps[0]["seed"] >> 32 == 7
    third, rs = adamw(bits=8, seed=3)
    third.load_state_dict({k: v for k, v in saved.items() if k in ("state", "param_groups")})
    assert third.seed == 3 and third.state[rs[0]]["step"] == 1
    for bad in (-1, 1 << 32, None, 0.5):
        before = _snapshot(third, rs)
        with pytest.raises(ValueError, match="seed"):
            third.load_state_dict({**saved, "seed": bad})
        _unchanged(third, rs, before)
        assert third.seed == 3
