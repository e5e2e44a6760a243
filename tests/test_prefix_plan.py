"""The plan of oda_prefix_decode_attn: what it was made for, and the sizes at which
its workgroup goes more than one round."""
import numpy as np
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


def _items(p):
    """Items of the plan (word 7 of its header)."""
    return int(p.plan[:32].view(torch.int32)[7].item())


# groups, heads and layers, whether the items are listed by their cost (more than one per CU)
LARGE = {
    "items of more than one round": (dict(groups=[(40, [5 + 37 * i for i in range(20)]), (7, [600, 20, 300])], Hq=64, Hkv=4,
                                          D=64, L=4), True),
    "many units": (dict(groups=[(3, [10, 200, 33]), (0, [90])], Hq=32, Hkv=8, D=64, L=20), True),
    "several tokens, two chunks": (dict(groups=[(60, [1 + 29 * i for i in range(9)])], Hq=48, Hkv=3, D=128, L=6, T=3), True),
    "300 requests, 150 groups": (dict(groups=[(j % 4, [1 + (7 * j) % 50, 3 + j % 20]) for j in range(150)], Hq=2, Hkv=1,
                                      D=64), True),
    "600 requests of one group": (dict(groups=[(5, [1 + i % 70 for i in range(600)])], Hq=4, Hkv=2, D=64), True),
    "2048 requests, a group each": (dict(groups=[(j % 3, [1 + j % 37]) for j in range(2048)], Hq=1, Hkv=1, D=64, spare=0), True),
    "2048 requests, two groups": (dict(groups=[(2, [1 + j % 20 for j in range(1500)]), (1, [1 + j % 30 for j in range(548)])],
                                       Hq=2, Hkv=1, D=64, spare=0), True),
    "200 groups, few with members": (dict(groups=[(2, [9, 30]) if j % 40 == 7 else (1, []) for j in range(200)], Hq=4, Hkv=2,
                                          D=64), False),
}


@pytest.mark.parametrize("cur", [True, False])
@pytest.mark.parametrize("name", LARGE)
def test_large_plans_match_oracle(name, cur):
    kw, by_cost = LARGE[name]
    p = Problem(62, cur=cur, **kw)
    p.upload()
    got = p.run()
    assert (p.L * p.Hkv * _items(p) > 256) == by_cost
    p.check(got)
    again = p.run()                                 # (items of like cost come in any order; results do not change)
    for a, b in zip(got, again):
        np.testing.assert_array_equal(a, b)


def test_flags_and_counts_of_many_requests():
    """Rows that are left alone among 500 requests, lengths out of range among the rest."""
    g = np.random.default_rng(63)
    p = Problem(63, [(j % 5, [1 + int(g.integers(0, 60)) for _ in range(1 + j % 6)]) for j in range(140)], 4, 2, 64, T=3,
                tokens=g.integers(-1, 5, size=97), spare=7)
    p.flags = g.integers(0, 2, size=p.B).astype(np.int32)
    bad = [b for b in p.members[::31] if p.flags[b]]
    for b in bad:
        p.seq[b] = p.max_len + 1 + b
    p.upload()
    p.check(nan=bad)


def test_order_of_members_changes_roundings_only():
    p = Problem(64, [(30, [10, 200, 31, 5]), (2, [90, 3])], 8, 2, 128, T=3, L=2)
    p.upload()
    out, lse = p.run()
    p.members[:4] = p.members[:4][::-1]
    p.upload()
    out2, lse2 = p.run()
    rows = p.attended()
    # weights and sums are off by about 2e-7 (tests/test_prefix_values.py), exponents of |lse| < 8 by 2^-22
    assert np.linalg.norm(out[:, rows] - out2[:, rows]) <= 1e-6 * np.linalg.norm(out[:, rows])
    np.testing.assert_allclose(lse[:, rows], lse2[:, rows], rtol=0, atol=2e-6)
