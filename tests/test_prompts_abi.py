"""Refusals of the operators that take prompts in: host-visible arguments are checked
before anything touches the GPU (no device work is needed)."""
import ctypes

import pytest

from test_abi import L  # noqa: F401  (the library's binding)

A = 1 << 20          # stands for an aligned device address (never dereferenced on a refusal)


def shape(L, **kw):
    base = dict(num_layers=1, batch=3, num_q_heads=8, num_kv_heads=2, head_dim=128, max_blocks_per_seq=4, max_seq_len=64,
                num_blocks=20)
    base.update(kw)
    return L.Shape(**base)


def refused(L, status, fn, *args):
    with pytest.raises(L.OdaError) as e:
        fn(*args)
    assert e.value.status == status, e.value
    assert e.value.detail


@pytest.mark.parametrize("kw,rows,status", [
    (dict(num_layers=2), 5, -2), (dict(split_blocks=2), 5, -2), (dict(batch=2049), 5, -3), (dict(), 0, -2), (dict(), -4, -2),
    (dict(head_dim=96), 5, -3), (dict(num_q_heads=7), 5, -2), (dict(), 2 ** 31 - 1, -2)])
def test_sizes(L, kw, rows, status):
    r = L.prompt_rows(rows, A)
    refused(L, status, L.prompt_plan_size, shape(L, **kw), r)
    refused(L, status, L.prompt_workspace_size, shape(L, **kw), r)
    refused(L, status, lambda: L.prompt_plan(shape(L, **kw), r, A, True, 0, A, 1 << 40, 0))


def test_sizes_grow_with_rows(L):
    sizes = [(L.prompt_plan_size(shape(L), L.prompt_rows(n, A)), L.prompt_workspace_size(shape(L), L.prompt_rows(n, A)))
             for n in (1, 100, 10000)]
    assert sizes[0] <= sizes[1] <= sizes[2] and all(p % 256 == 0 and w % 256 == 0 for p, w in sizes)


def test_plan(L):
    s, r = shape(L), L.prompt_rows(9, A)
    n = L.prompt_plan_size(s, r)
    plan = lambda *a: L.prompt_plan(*a, stream=0)  # noqa: E731
    refused(L, -1, plan, s, r, None, True, 0, A, n)
    refused(L, -1, plan, s, L.prompt_rows(9, None), A, True, 0, A, n)
    refused(L, -2, plan, s, r, A, True, -1, A, n)
    refused(L, -2, plan, s, r, A, False, 5, A, n)                 # a window without the causal mask
    refused(L, -4, plan, s, r, A, True, 0, None, n)
    refused(L, -4, plan, s, r, A, True, 0, A, n - 1)
    refused(L, -4, plan, s, r, A, True, 0, A + 16, n)
    assert L._lib.oda_prompt_plan(ctypes.byref(s.c()), ctypes.byref(r), A, 2, 0, A, n, 0) == -2
    assert L._lib.oda_prompt_plan(None, ctypes.byref(r), A, 1, 0, A, n, 0) == -1
    assert L._lib.oda_prompt_plan(ctypes.byref(s.c()), None, A, 1, 0, A, n, 0) == -1


def test_attention(L):
    s, r = shape(L), L.prompt_rows(9, A)
    n, w = L.prompt_plan_size(s, r), L.prompt_workspace_size(s, r)

    def call(plan=A, plan_bytes=n, out=A, out_type=0, ws=A, ws_bytes=w, sh=s, rows=r, **kw):
        a = dict(q=A, k_cache=A, v_cache=A, block_table=A, seq_lens=None, scale=0.1, k_cur=None, v_cur=None)
        a.update(kw)
        cs, inp = sh.c(), L.inputs(a["q"], a["k_cache"], a["v_cache"], a["block_table"], a["seq_lens"], a["scale"], a["k_cur"],
                                   a["v_cur"])
        return L._lib.oda_prompt_attn(ctypes.byref(cs), ctypes.byref(inp), ctypes.byref(rows), plan, plan_bytes, out, out_type,
                                      None, ws, ws_bytes, 0)

    for name in ("q", "k_cache", "v_cache", "block_table"):
        assert call(**{name: None}) == -1
    assert call(out=None) == -1
    assert call(k_cur=A, v_cur=A) == -2
    assert call(out_type=2) == -2 and call(out_type=-1) == -2
    for name in ("q", "k_cache", "v_cache"):
        assert call(**{name: A + 8}) == -2
    assert call(out=A + 4) == -2
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert call(scale=scale) == -2
    assert call(plan=None) == -4 and call(plan_bytes=n - 1) == -4 and call(plan=A + 128) == -4
    assert call(ws=None) == -4 and call(ws_bytes=w - 1) == -4 and call(ws=A + 128) == -4
    assert call(sh=shape(L, num_layers=2)) == -2
    assert L._lib.oda_prompt_attn(ctypes.byref(s.c()), None, ctypes.byref(r), A, n, A, 0, None, A, w, 0) == -1


def append(L, status, sh=None, rows=9, start=A, seq=A, kv=(A, A), table=A, q=A, rings=(None, None, 0, 0), **kw):
    a = dict(qkv=A, q_gain=A, k_gain=A, rms_eps=1e-6, rope_theta=1e4, positions=None, num_axes=1, axis_pairs=(0, 0, 0, 0), type=0)
    a.update(kw)
    d = L.AppendDesc(a["qkv"], a["type"], a["rms_eps"], a["q_gain"], a["k_gain"], a["rope_theta"], a["positions"], a["num_axes"],
                     (ctypes.c_int32 * 4)(*a["axis_pairs"]))
    cs, r = (sh or shape(L)).c(), L.prompt_rows(rows, start)
    got = L._lib.oda_append_qkv(ctypes.byref(cs), ctypes.byref(r), ctypes.byref(d), *kv, table, seq, q, *rings, 0)
    assert got == status, (got, L.last_error())
    assert L.last_error()


def test_append(L):
    append(L, -2, sh=shape(L, num_layers=2))
    append(L, -3, sh=shape(L, head_dim=32))
    append(L, -2, rows=0)
    append(L, -1, start=None)
    append(L, -1, seq=None)
    append(L, -1, qkv=None)
    append(L, -1, kv=(A, None))
    append(L, -1, kv=(None, None), q=None)
    append(L, -1, table=None)
    append(L, -1, rings=(A, None, 4, 64))
    append(L, -1, kv=(None, None), rings=(A, A, 4, 64))
    append(L, -2, rings=(A, A, -1, 64))
    append(L, -2, rings=(A, A, 4, 0))
    append(L, -2, type=2)
    for theta in (1.0, -2.0, 0.5, float("inf"), float("nan")):
        append(L, -2, rope_theta=theta)
    for eps in (-1.0, float("inf"), float("nan")):
        append(L, -2, rms_eps=eps)
    append(L, -2, num_axes=0)
    append(L, -2, num_axes=5)
    append(L, -1, num_axes=3, axis_pairs=(22, 21, 21, 0))
    append(L, -2, num_axes=3, axis_pairs=(22, 21, 20, 0), positions=A)
    append(L, -2, num_axes=2, axis_pairs=(-1, 65, 0, 0), positions=A)
    for name in ("qkv", "q_gain", "k_gain", "q"):
        append(L, -2, **{name: A + 8})
    append(L, -2, kv=(A + 2, A))
    append(L, -2, rings=(A, A + 2, 4, 64))
    s = shape(L).c()
    d = L.append_desc(A, None, None, 0.0, 0.0)
    r = L.prompt_rows(3, A)
    assert L._lib.oda_append_qkv(None, ctypes.byref(r), ctypes.byref(d), A, A, A, A, A, None, None, 0, 0, 0) == -1
    assert L._lib.oda_append_qkv(ctypes.byref(s), None, ctypes.byref(d), A, A, A, A, A, None, None, 0, 0, 0) == -1
    assert L._lib.oda_append_qkv(ctypes.byref(s), ctypes.byref(r), None, A, A, A, A, A, None, None, 0, 0, 0) == -1


def test_logprobs(L):
    for kw, rows, status in ((dict(vocab=0), 1, -2), (dict(vocab=2 ** 30 + 1), 1, -2), (dict(top=-1), 1, -2), (dict(top=33), 1, -2),
                             (dict(row_stride=9), 1, -2), (dict(row_stride=-10), 1, -2), (dict(), 0, -2)):
        a = dict(vocab=10, top=2, logits=A, tokens=A, row_stride=0)
        a.update(kw)
        refused(L, status, L.logprob_workspace_size, L.logprob_desc(**a), rows)
    d = L.logprob_desc(10, 2, A, A)
    n = L.logprob_workspace_size(d, 4)
    call = lambda d, *a, ws=A, size=n, lists=(None, None): L.token_logprobs(d, 4, *a, ws, *lists, size, 0)  # noqa: E731
    refused(L, -1, call, L.logprob_desc(10, 2, None, A), A, A, A, A, A)
    refused(L, -1, call, L.logprob_desc(10, 2, A, None), A, None, A, A, A)
    refused(L, -1, call, L.logprob_desc(10, 2, A, None), None, A, A, A, A)
    refused(L, -1, call, d, A, A, A, None, A)
    refused(L, -1, call, d, A, A, A, A, None)
    refused(L, -1, call, L.logprob_desc(10, 0, A, A), A, A, A, A, A)
    refused(L, -1, call, L.logprob_desc(10, 0, A, A), None, None, None, None, None)
    refused(L, -1, lambda: call(d, A, A, A, A, A, lists=(A, None)))
    refused(L, -4, lambda: call(d, A, A, A, A, A, ws=None))
    refused(L, -4, lambda: call(d, A, A, A, A, A, size=n - 1))
    refused(L, -4, lambda: call(d, A, A, A, A, A, ws=A + 64))
    assert L._lib.oda_token_logprobs(None, 4, A, A, A, A, A, None, None, A, n, 0) == -1
    assert L._lib.oda_logprob_workspace_size(None, 4, ctypes.byref(ctypes.c_size_t())) == -1


def test_binding_checks(L):
    with pytest.raises(ValueError):
        L.append_desc(A + 0, None, None, 0.0, 0.0, A, [1, 2, 3, 4, 5])
