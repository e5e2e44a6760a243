"""Argument checks of the adapter, verification and draft-commit entry points
(no device work: every refusal comes before a launch), and their workspace
sizes."""
import os

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2609_20734_amd import build as B
    if not os.path.exists(B.LIB):
        B.build()
    import paper_2609_20734_amd._lib as lib
    return lib


def status_of(L, fn):
    with pytest.raises(L.OdaError) as e:
        fn()
    assert L.last_error()
    return e.value.status


def test_lora_workspace_size(L):
    d = L.lora_desc(4, 16, [100, 50, 50], 0x1000, 0x2000, 0x3000)
    assert L.lora_workspace_size(d, 1) >= 48 * 4 and L.lora_workspace_size(d, 33) >= 33 * 48 * 4
    assert L.lora_workspace_size(d, 33) % 256 == 0
    assert status_of(L, lambda: L.lora_workspace_size(d, 0)) == -2
    for bad, status in [((0, 16, [4]), -2), ((1, 0, [4]), -3), ((1, 12, [4]), -3), ((1, 136, [4]), -3), ((1, -8, [4]), -3),
                        ((1, 16, [4, 0]), -2)]:
        assert status_of(L, lambda: L.lora_workspace_size(L.lora_desc(*bad, 0x1000, 0x2000, 0x3000), 1)) == status
    with pytest.raises(ValueError):
        L.lora_desc(1, 8, [], 0x1000, 0x2000, 0x3000)
    with pytest.raises(ValueError):
        L.lora_desc(1, 8, [1, 1, 1, 1, 1], 0x1000, 0x2000, 0x3000)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), -1), (dict(y=None), -1), (dict(ids=None), -1), (dict(a=None), -1), (dict(b=None), -1),
    (dict(scale=None), -1), (dict(work=0x9000), -1), (dict(batch=0), -2), (dict(parts=[32, 31]), -2),
    (dict(parts=[64, 64]), -2), (dict(a=0x1008), -2), (dict(b=0x2004), -2), (dict(K=60), -2),
    (dict(rank=12), -3), (dict(ws=None), -4), (dict(wb=255), -4), (dict(ws=0x100010), -4), (dict(batch=1 << 17), -4),
    (dict(swiglu=True), -2), (dict(swiglu=True, parts=[64, 64], residual=0x7000), -3), (dict(x=0x5004), -2)])
def test_lora_refusals(L, kw, status):
    a = dict(K=64, parts=[32, 32], rank=16, batch=2, x=0x5000, y=0x6000, ids=0x8000, a=0x1000, b=0x2000, scale=0x3000,
             ws=0x100000, wb=256, residual=None, swiglu=False, work=None)
    a.update(kw)
    desc = L.dense_desc(a["K"], 64, L.DENSE_SWIGLU if a["swiglu"] else L.DENSE_PLAIN, 0x4000)
    lora = L.lora_desc(3, a["rank"], a["parts"], a["a"], a["b"], a["scale"])
    assert status_of(L, lambda: L.dense_lora_bf16(desc, lora, a["batch"], a["x"], a["residual"], a["y"], a["ids"], a["ws"],
                                                  a["work"], None, a["wb"], stream=0)) == status


def test_verify_workspace_size(L):
    one = L.verify_workspace_size(1, 1000, 4)
    assert one % 256 == 0
    assert L.verify_workspace_size(8, 1000, 4) > one and L.verify_workspace_size(1, 1000, 5) >= one
    for V in (1, 4096, 151936, 1 << 30):
        assert L.verify_workspace_size(1, V, 4) == one       # splits are bounded: the vocabulary does not count
    for bad in [(0, 10, 1), (1, 0, 1), (1, 10, -1), (1, 10, 64), (1, (1 << 30) + 1, 1), (65536, 10, 1)]:
        assert status_of(L, lambda: L.verify_workspace_size(*bad)) == -2


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), -1), (dict(u=None), -1), (dict(acc=None), -1), (dict(tok=None), -1), (dict(x=None), -1),
    (dict(n_work=0x9000), -1), (dict(batch=0), -2), (dict(V=0), -2), (dict(K=64), -2), (dict(K=-1), -2),
    (dict(ws=None), -4), (dict(short=1), -4), (dict(ws=0x100020), -4)])
def test_verify_refusals(L, kw, status):
    a = dict(V=1000, K=3, logits=0x1000, x=0x2000, u=0x3000, acc=0x4000, tok=0x5000, ws=0x100000, short=0, batch=2,
             n_work=None)
    a.update(kw)
    wb = L.verify_workspace_size(2, 1000, 3) - a["short"]
    d = L.verify_desc(a["V"], a["K"], a["logits"], a["x"], a["u"])
    assert status_of(L, lambda: L.verify_drafts(d, a["batch"], a["acc"], a["tok"], a["ws"], None, a["n_work"], wb,
                                                stream=0)) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), -1), (dict(kc=None), -1), (dict(vc=None), -1), (dict(seq=None), -1), (dict(k_ring=0x9000), -1),
    (dict(T=0), -2), (dict(T=65), -2), (dict(kc=0x5008), -2), (dict(rows=0xa000, advance=False), -2),
    (dict(k_ring=0x9000, v_ring=0xb000), -2), (dict(k_ring=0x9000, v_ring=0xb000, n_sink=-1, window=4), -2),
    (dict(k_ring=0x9001, v_ring=0xb000, window=4), -2),
    (dict(ws=None), -4), (dict(wb=255), -4), (dict(ws=0x100010), -4), (dict(head_dim=96), -3), (dict(batch=0), -2),
    (dict(num_layers=1 << 24), -2)])
def test_commit_drafts_refusals(L, kw, status):
    a = dict(T=4, k=0x1000, v=0x2000, table=0x3000, seq=0x4000, kc=0x5000, vc=0x6000, ws=0x100000, wb=256, advance=True,
             rows=None, k_ring=None, v_ring=None, n_sink=0, window=0, head_dim=64, batch=3, num_layers=2)
    a.update(kw)
    shape = L.Shape(a["num_layers"], a["batch"], 2, 2, a["head_dim"], 4, 64, 12)
    assert status_of(L, lambda: L.commit_drafts(shape, a["T"], a["k"], a["v"], a["table"], a["seq"], a["kc"], a["vc"], None,
                                                a["advance"], a["rows"], a["ws"], a["k_ring"], a["v_ring"], a["n_sink"],
                                                a["window"], a["wb"], stream=0)) == status


def _prefix_shape(L, **kw):
    base = dict(num_layers=2, batch=3, num_q_heads=8, num_kv_heads=2, head_dim=128, max_blocks_per_seq=4, max_seq_len=64,
                num_blocks=20)
    base.update(kw)
    return L.Shape(**base)


def _prefix_groups(L, NG=2, T=4, start=0x1000, members=0x2000, blocks=0x3000):
    return L.prefix_groups(NG, T, start, members, blocks)


def test_prefix_sizes(L):
    s, g = _prefix_shape(L), _prefix_groups(L)
    plan, ws = L.prefix_plan_size(s, g), L.prefix_workspace_size(s, g)
    assert plan % 256 == 0 and ws % 256 == 0
    assert L.prefix_plan_size(_prefix_shape(L, batch=300), g) > plan
    assert L.prefix_workspace_size(_prefix_shape(L, batch=300), g) > ws
    for kw, gw, status in [(dict(batch=2049), {}, -3), (dict(head_dim=96), {}, -3), (dict(batch=0), {}, -2),
                           (dict(split_blocks=2), {}, -2), (dict(num_q_heads=34), {}, -3), ({}, dict(T=0), -2),
                           ({}, dict(T=17), -2), ({}, dict(NG=0), -2), ({}, dict(NG=2049), -2)]:
        assert status_of(L, lambda: L.prefix_plan_size(_prefix_shape(L, **kw), _prefix_groups(L, **gw))) == status
        assert status_of(L, lambda: L.prefix_workspace_size(_prefix_shape(L, **kw), _prefix_groups(L, **gw))) == status


@pytest.mark.parametrize("kw,status", [
    (dict(seq=None), -1), (dict(start=None), -1), (dict(members=None), -1), (dict(blocks=None), -1), (dict(kc=0x8000), -1),
    (dict(plan=None), -4), (dict(short=1), -4), (dict(plan=0x200040), -4)])
def test_prefix_plan_refusals(L, kw, status):
    a = dict(seq=0x5000, start=0x1000, members=0x2000, blocks=0x3000, kc=None, plan=0x200000, short=0)
    a.update(kw)
    s, g = _prefix_shape(L), _prefix_groups(L, start=a["start"], members=a["members"], blocks=a["blocks"])
    inp = L.inputs(None, None, None, None, a["seq"], 0.1, a["kc"], None)
    n = L.prefix_plan_size(s, g) - a["short"]
    assert status_of(L, lambda: L.prefix_plan(s, inp, g, a["plan"], n, stream=0)) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), -1), (dict(k=None), -1), (dict(table=None), -1), (dict(out=None), -1), (dict(kc=0x8000), -1),
    (dict(q=0x4008), -2), (dict(kc=0x8008, vc=0x9000), -2), (dict(scale=0.0), -2), (dict(scale=float("nan")), -2),
    (dict(out=0xa004), -2), (dict(plan=None), -4), (dict(short_plan=1), -4), (dict(ws=None), -4), (dict(short=1), -4),
    (dict(ws=0x300010), -4)])
def test_prefix_attention_refusals(L, kw, status):
    a = dict(q=0x4000, k=0x5000, v=0x6000, table=0x7000, kc=None, vc=None, scale=0.1, out=0xa000, plan=0x200000,
             ws=0x300000, short=0, short_plan=0)
    a.update(kw)
    s, g = _prefix_shape(L), _prefix_groups(L)
    inp = L.inputs(a["q"], a["k"], a["v"], a["table"], None, a["scale"], a["kc"], a["vc"])
    pn, wn = L.prefix_plan_size(s, g) - a["short_plan"], L.prefix_workspace_size(s, g) - a["short"]
    assert status_of(L, lambda: L.prefix_decode_attn(s, inp, g, a["plan"], a["out"], None, a["ws"], pn, wn,
                                                     stream=0)) == status
