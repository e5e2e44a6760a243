"""The plan of oda_prefix_decode_attn: what it was made for, and the sizes at which
its workgroup goes more than one round."""
import pytest
import torch

from test_prefix import Problem

pytestmark = pytest.mark.gpu


def _groups(p, count):
    """The problem's arrays under another num_groups."""
    return p.P.prefix_groups(count, p.T, p.dstart, p.dmembers, p.dprefix, p.dtok, p.dflags)


@pytest.mark.parametrize("other", [1, 7, 9])
def test_a_plan_of_another_group_count_gives_nan(other):
    """Eight groups of a block each in 224 (layer, KV head) units: 16 items, more than a call with one group launches."""
    p = Problem(61, [(1, [3 + i]) for i in range(8)], 32, 8, 64, L=28, spare=0)
    p.start += [len(p.members)] * 2                 # (empty groups, so that nine can be named)
    p.prefix += [0, 0]
    p.upload()
    eight, others = _groups(p, 8), _groups(p, other)
    size = max(p.P.prefix_plan_size(p.shape, g) for g in (eight, others))
    plan = torch.zeros(size, dtype=torch.uint8, device="cuda")
    ws = torch.zeros(max(p.P.prefix_workspace_size(p.shape, g) for g in (eight, others)), dtype=torch.uint8, device="cuda")
    for made, called in ((eight, others), (others, eight)):
        p.out.fill_(-7.0)
        p.lse.fill_(-7.0)
        p.P.prefix_plan(p.shape, p.inp, made, plan)
        p.P.prefix_decode_attn(p.shape, p.inp, called, plan, p.out, p.lse, ws)
        torch.cuda.synchronize()
        assert torch.isnan(p.out).all() and torch.isnan(p.lse).all()
    p.groups, p.plan, p.ws = eight, plan, ws
    p.check()
