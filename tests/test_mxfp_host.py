"""The host side of the calls on pools in four bits, without a GPU: refusals of parameters and arguments, the binding's own checks."""
import ctypes

import pytest
import torch

from paper_2410_16179_amd import binding as mp
from tests.test_paged_host import FAKE, INVALID, LAUNCH, OK, SMALL, UNSUPPORTED, accepted, posing

BLOCKS = ("k_block_scales", "v_block_scales")


def params(**kw):
    return mp.make_paged_params(**{**dict(batch=3, n_q_heads=8, n_kv_heads=2, dtype="bf16", kv_dtype="mxfp4", page_size=16, max_pages=40, n_pages=100,
                                          max_tokens=12, max_new=4), **kw})


def append(p, **kw):
    names = ["k_new", "v_new", "slots", "k_pages", "v_pages", *BLOCKS]
    at = {n: FAKE for n in names} | kw
    return mp.lib().magicpig_page_append_mxfp(p if p is None else ctypes.byref(p), *[at[n] for n in names], None)


def read(p, **kw):
    names = ["k_pages", "v_pages", *BLOCKS, "slots", "k_out", "v_out"]
    at = {n: FAKE for n in names} | kw
    return mp.lib().magicpig_page_read_mxfp(p if p is None else ctypes.byref(p), *[at[n] for n in names], None)


def attend(p, **kw):
    names = ["q", "k_pages", "v_pages", *BLOCKS, "block_table", "lengths", "token_start", "out", "lse"]
    at = {n: FAKE for n in names} | {"workspace": FAKE, "bytes": 1 << 40} | kw
    return mp.lib().magicpig_paged_attention_mxfp(p if p is None else ctypes.byref(p), *[at[n] for n in names], at["workspace"], at["bytes"], None)


CALLS = (append, read, attend)


@pytest.mark.parametrize("field,value,status", [("batch", -1, INVALID), ("head_dim", 64, UNSUPPORTED), ("dtype", mp.MAGICPIG_FP32, UNSUPPORTED),
                                                ("page_size", 24, UNSUPPORTED), ("n_pages", 0, INVALID), ("max_tokens", 0, INVALID), ("max_new", 0, INVALID),
                                                ("kv_dtype", 3, UNSUPPORTED), ("kv_dtype", 5, UNSUPPORTED)])
def test_parameters(field, value, status):
    p = params()
    setattr(p, field, value)
    assert [call(p) for call in CALLS] == [status] * 3
    assert mp.magicpig_paged_workspace_bytes(p) == 0
    assert [call(None) for call in CALLS] == [INVALID] * 3


@pytest.mark.parametrize("kv", ["", "fp8"])
def test_pools_of_other_kinds(kv):
    assert [call(params(kv_dtype=kv)) for call in CALLS] == [UNSUPPORTED] * 3


def test_the_calls_on_other_pools_refuse_these():
    p = ctypes.byref(params())
    assert mp.lib().magicpig_page_append(p, FAKE, FAKE, FAKE, None, None, FAKE, FAKE, None) == UNSUPPORTED
    assert mp.lib().magicpig_paged_attention(p, FAKE, FAKE, FAKE, None, None, FAKE, FAKE, None, FAKE, None, FAKE, 1 << 40, None) == UNSUPPORTED


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("part,value,status", [("page", -128, INVALID), ("key", 64, INVALID), ("key", 0, INVALID), ("head", -128, INVALID),
                                               ("page", 64, UNSUPPORTED), ("key", 160, UNSUPPORTED), ("head", 192, UNSUPPORTED),
                                               ("key", 1 << 28, UNSUPPORTED), ("key", 1 << 40, UNSUPPORTED)])
def test_pool_strides(which, part, value, status):
    p = params()
    setattr(p, f"{which}_stride_{part}", value)
    assert [call(p) for call in CALLS] == [status] * 3


def test_strides_of_token_arrays():
    for name, calls in (("q", (attend,)), ("k_new", (append, read)), ("v_new", (append, read))):
        for part, value, status in (("token", -8, INVALID), ("head", -8, INVALID), ("token", 4, UNSUPPORTED), ("head", 12, UNSUPPORTED)):
            p = params()
            setattr(p, f"{name}_stride_{part}", value)
            assert [call(p) for call in calls] == [status] * len(calls)


def test_missing_and_misaligned_arguments():
    p = params()
    for call, names in ((append, ("k_new", "v_new", "slots", "k_pages", "v_pages", *BLOCKS)), (read, ("k_pages", "v_pages", *BLOCKS, "slots", "k_out", "v_out")),
                        (attend, ("q", "k_pages", "v_pages", *BLOCKS, "block_table", "lengths", "out"))):
        for name in names:
            assert call(p, **{name: None}) == INVALID, name
            assert call(p, **{name: FAKE + 2}) == INVALID, name
    for name in ("token_start", "lse"):
        assert attend(p, **{name: FAKE + 2}) == INVALID
    assert attend(p, workspace=FAKE + 8) == INVALID
    assert attend(params(batch=13), token_start=None) == INVALID
    assert attend(p, bytes=255) == attend(p, workspace=None) == SMALL


@accepted
def test_what_is_accepted_gets_as_far_as_the_launch():
    p = params(max_pages=2000)
    assert append(p) == read(p) == attend(p) == attend(p, lse=None, token_start=None) == LAUNCH
    assert attend(p, bytes=mp.magicpig_paged_workspace_bytes(p)) == LAUNCH
    assert append(p, k_block_scales=FAKE + 4) == LAUNCH
    assert attend(params(max_new=1 << 24)) == LAUNCH
    assert attend(params(batch=0), block_table=None, lengths=None) == OK
    names = [FAKE] * 10
    assert mp.lib().magicpig_page_plan(ctypes.byref(p), *names, FAKE, 1 << 30, None) == LAUNCH


def arguments(p, bytes_=torch.uint8):
    bf = torch.bfloat16
    pool, block = posing(p.n_pages, 16, 2, 64, dtype=bytes_), posing(p.n_pages, 16, 2, 4, dtype=torch.uint8)
    rows = posing(p.max_tokens, 2, 128, dtype=bf)
    return {"append": [rows, rows, posing(p.max_tokens, dtype=torch.int64), pool, pool, block, block],
            "read": [pool, pool, block, block, posing(p.max_tokens, dtype=torch.int64), rows, rows],
            "attend": [posing(p.max_tokens, 8, 128, dtype=bf), pool, pool, block, block, posing(3, p.max_pages), posing(3), posing(4),
                       posing(p.max_tokens, 8, 128, dtype=bf), posing(p.max_tokens, 8, dtype=torch.float32)]}


BOUND = {"append": mp.magicpig_page_append_mxfp, "read": mp.magicpig_page_read_mxfp, "attend": mp.magicpig_paged_attention_mxfp}


@pytest.mark.parametrize("which,at,tensor,says", [
    ("append", 0, lambda: posing(12, 1, 128, dtype=torch.bfloat16), "k_new"), ("append", 3, lambda: posing(100, 16, 2, 63, dtype=torch.uint8), "k_pages"),
    ("append", 4, lambda: posing(100, 16, 2, 64, dtype=torch.bfloat16), "v_pages"), ("append", 5, lambda: posing(100, 16, 2, 3, dtype=torch.uint8), "k_block_scales"),
    ("append", 6, lambda: None, "v_block_scales"), ("append", 2, lambda: posing(12), "slots"), ("read", 3, lambda: posing(99, 16, 2, 4, dtype=torch.uint8), "v_block_scales"),
    ("read", 5, lambda: posing(12, 2, 128, dtype=torch.float32), "k_out"), ("read", 6, lambda: posing(11, 2, 128, dtype=torch.bfloat16), "v_out"),
    ("attend", 3, lambda: posing(100, 16, 2, 4, dtype=torch.float32), "k_block_scales"), ("attend", 2, lambda: posing(100, 16, 2, 64, dtype=torch.uint8, device=1), "device"),
    ("attend", 5, lambda: posing(3, 39), "block_table"), ("attend", 8, lambda: posing(12, 8, 127, dtype=torch.bfloat16), "out")])
def test_binding_refuses_tensors_that_do_not_fit(which, at, tensor, says):
    p = params()
    got = arguments(p)[which]
    got[at] = tensor()
    with pytest.raises(mp.MagicpigError, match=says):
        BOUND[which](p, *got)
    with pytest.raises(mp.MagicpigError, match="MXFP4"):
        BOUND[which](params(kv_dtype="fp8"), *arguments(p)[which])


def test_binding_passes_on_what_fits(monkeypatch):
    calls = []
    monkeypatch.setattr(mp, "_paged_call", lambda *a: calls.append(a))
    p = params()
    for dtype in (torch.uint8, torch.float4_e2m1fn_x2):
        for which, got in arguments(p, torch.uint8).items():
            if dtype is not torch.uint8:
                got = [t.view(dtype) if t.dtype is torch.uint8 and t.shape[-1] == 64 else t for t in got]
            BOUND[which](p, *got)
    assert len(calls) == 6 and all(a[2]._obj is p for a in calls)
