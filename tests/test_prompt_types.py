"""Types of projections and outputs through the binding: a tensor's own, or, for a plain
address, the one that is given.  No device work is needed."""
import pytest
import torch

from test_abi import L  # noqa: F401  (the library's binding)

A = 1 << 20          # stands for an aligned device address (never dereferenced)


def out_type(L, out, **kw):
    s, r = L.Shape(1, 3, 8, 2, 128, 4, 64, 20), L.prompt_rows(9, A)
    return L.prepare_prompt_attn(s, L.inputs(A, A, A, A, None, 0.1), r, A, out, None, A, 1, 1, 0, **kw).args[6]


@pytest.mark.parametrize("dtype,name", [(torch.float32, "F32"), (torch.bfloat16, "BF16"), (torch.int16, "BF16"),
                                        (torch.uint16, "BF16")])
def test_a_tensor_has_its_own(L, dtype, name):
    t, kind = torch.zeros(8, dtype=dtype), getattr(L, name)
    other = L.F32 + L.BF16 - kind
    assert out_type(L, t) == out_type(L, t, out_type=kind) == kind
    assert L.append_desc(t, None, None, 0.0, 0.0).qkv_type == L.append_desc(t, None, None, 0.0, 0.0, qkv_type=kind).qkv_type == kind
    with pytest.raises(ValueError):
        out_type(L, t, out_type=other)
    with pytest.raises(ValueError):
        L.append_desc(t, None, None, 0.0, 0.0, qkv_type=other)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.int32])
def test_other_tensors_are_refused(L, dtype):
    t = torch.zeros(8, dtype=dtype)
    with pytest.raises(ValueError):
        out_type(L, t)
    with pytest.raises(ValueError):
        L.append_desc(t, None, None, 0.0, 0.0)


def test_an_address_has_the_one_given(L):
    assert out_type(L, A) == L.F32 and out_type(L, A, out_type=L.BF16) == L.BF16
    assert L.append_desc(A, None, None, 0.0, 0.0).qkv_type == L.F32
    assert L.append_desc(A, None, None, 0.0, 0.0, qkv_type=L.BF16).qkv_type == L.BF16


def test_unknown_types_are_refused(L):
    s, r = L.Shape(1, 3, 8, 2, 128, 4, 64, 20), L.prompt_rows(9, A)
    n, w = L.prompt_plan_size(s, r), L.prompt_workspace_size(s, r)
    with pytest.raises(L.OdaError) as e:
        L.prompt_attn(s, L.inputs(A, A, A, A, None, 0.1), r, A, A, None, A, n, w, 0, out_type=7)
    assert e.value.status == -2
    with pytest.raises(L.OdaError) as e:
        L.append_qkv(s, r, L.append_desc(A, None, None, 0.0, 0.0, qkv_type=7), A, A, A, A, A, stream=0)
    assert e.value.status == -2
