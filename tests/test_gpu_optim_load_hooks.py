"""Loading a state calls the hooks that torch's optimizers have for it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def optimizer(**kw):
    from paper_2604_10103_b200 import optim
    p = torch.nn.Parameter(torch.ones(300, device="cuda"))
    p.grad = torch.ones_like(p)
    return optim.AdamW([p], **kw), p


def test_hooks_before_and_after():
    opt, p = optimizer(lr=0.5)
    saved, _ = optimizer(lr=0.25)
    saved.step()
    state, calls = saved.state_dict(), []

    def before(o, s):
        calls.append(("before", o is opt, o.param_groups[0]["lr"], int(o.state[p]["step"])))
        s["param_groups"] = [dict(s["param_groups"][0], lr=0.125)]      # (of a copy: the caller's own dictionary stays)

    def instead(o, s):
        calls.append(("instead", s["param_groups"][0]["lr"]))
        return dict(s, param_groups=[dict(s["param_groups"][0], weight_decay=0.75)])
    opt.register_load_state_dict_pre_hook(before)
    opt.register_load_state_dict_pre_hook(instead)
    handle = opt.register_load_state_dict_post_hook(lambda o: calls.append(("after", o.param_groups[0]["lr"], o.param_groups[0]["weight_decay"], int(o.state[p]["step"]))))
    opt.load_state_dict(state)
    assert calls == [("before", True, 0.5, 0), ("instead", 0.125), ("after", 0.125, 0.75, 1)]
    assert state["param_groups"][0]["lr"] == 0.25
    handle.remove()
    opt.load_state_dict(state)
    assert len(calls) == 5 and calls[3][0] == "before" and calls[4][0] == "instead"
