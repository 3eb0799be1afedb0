"""The host side of accounts and eviction, without a GPU: refusals of parameters and arguments, the binding's own checks, and the rules by which the
work is cut."""
import ctypes

import pytest
import torch

from paper_2410_16179_amd import binding as mp
from tests.test_paged_host import FAKE, INVALID, LAUNCH, OK, SMALL, UNSUPPORTED, accepted, params, posing

BLOCKS = ("k_block_scales", "v_block_scales")


def weigh(p, **kw):
    names = ["q", "k_pages", "k_scale", "k_block_scales", "block_table", "lengths", "token_start", "lse", "counted", "weights"]
    at = {n: FAKE for n in names} | {"k_scale": None, "k_block_scales": None, "workspace": None, "bytes": 0} | kw
    return mp.lib().magicpig_page_weights(p and ctypes.byref(p), *[at[n] for n in names], at["workspace"], at["bytes"], None)


def keep(p, **kw):
    at = {n: FAKE for n in ("weights", "block_table", "lengths", "budgets", "kept", "lengths_out")} | {
        "n_first": 4, "n_last": 9, "max_keep": 50, "workspace": FAKE, "bytes": 1 << 40} | kw
    return mp.lib().magicpig_page_keep(p and ctypes.byref(p), at["weights"], at["block_table"], at["lengths"], at["budgets"], at["n_first"], at["n_last"],
                                       at["max_keep"], at["kept"], at["lengths_out"], at["workspace"], at["bytes"], None)


def evict(p, **kw):
    names = ["lengths", "lengths_kept", "block_table", "free_pages", "n_free", "k_pages", "v_pages", *BLOCKS, "weights", "n_free_out", "status"]
    at = {n: FAKE for n in names} | {b: None for b in BLOCKS} | {"kept": FAKE, "max_keep": 50, "workspace": None, "bytes": 0} | kw
    return mp.lib().magicpig_page_evict(p and ctypes.byref(p), at["kept"], at["max_keep"], *[at[n] for n in names], at["workspace"], at["bytes"], None)


CALLS = (weigh, keep, evict)


@pytest.mark.parametrize("field,value,status", [("batch", -1, INVALID), ("head_dim", 64, UNSUPPORTED), ("dtype", 2, UNSUPPORTED), ("page_size", 24, UNSUPPORTED),
                                                ("n_pages", 0, INVALID), ("max_tokens", 0, INVALID), ("kv_dtype", 3, UNSUPPORTED)])
def test_parameters(field, value, status):
    p = params()
    setattr(p, field, value)
    assert [call(p) for call in CALLS] == [status] * 3
    assert [call(None) for call in CALLS] == [INVALID] * 3


def test_pool_and_row_strides():
    for name, calls in (("k", (weigh, evict)), ("v", (evict,))):
        for part, value, status in (("page", -8, INVALID), ("key", 120, INVALID), ("head", 12, UNSUPPORTED), ("key", 1 << 30, UNSUPPORTED)):
            p = params()
            setattr(p, f"{name}_stride_{part}", value)
            assert [call(p) for call in calls] == [status] * len(calls)
    for part, value, status in (("token", -8, INVALID), ("head", 4, UNSUPPORTED), ("token", (1 << 22) + 8, UNSUPPORTED), ("head", (1 << 22) + 8, UNSUPPORTED)):
        p = params()
        setattr(p, f"q_stride_{part}", value)
        assert weigh(p) == status


def test_missing_and_misaligned_arguments():
    p = params()
    for call, names in ((weigh, ("q", "k_pages", "block_table", "lengths", "lse", "weights")), (keep, ("weights", "block_table", "lengths", "budgets", "kept", "lengths_out")),
                        (evict, ("lengths", "lengths_kept", "block_table", "free_pages", "n_free", "k_pages", "v_pages", "n_free_out", "status"))):
        for name in names:
            assert call(p, **{name: None}) == INVALID, name
            assert call(p, **{name: FAKE + 2}) == INVALID, name
    for name in ("token_start", "counted"):
        assert weigh(p, **{name: FAKE + 2}) == INVALID
    assert keep(p, weights=FAKE + 4) == INVALID               # (read sixteen bytes at a time)
    for name in ("kept", "weights"):
        assert evict(p, **{name: FAKE + 2}) == INVALID
    for call in CALLS:
        assert call(p, workspace=FAKE + 8) == INVALID
    assert weigh(params(batch=13), token_start=None) == INVALID


def test_scales_belong_to_their_pools():
    assert weigh(params(), k_scale=FAKE) == INVALID and weigh(params(), k_block_scales=FAKE) == INVALID
    four = params(kv_dtype="mxfp4")
    assert weigh(four) == INVALID and weigh(four, k_block_scales=FAKE, k_scale=FAKE) == INVALID
    assert weigh(four, k_block_scales=FAKE + 2) == INVALID
    for b in BLOCKS:
        assert evict(params(), **{b: FAKE}) == INVALID
        assert evict(four, **{b: FAKE}) == INVALID            # (the other one is missing)
    assert evict(four, k_block_scales=FAKE, v_block_scales=FAKE + 2) == INVALID


def test_numbers():
    p = params()
    for name in ("n_first", "n_last"):
        assert keep(p, **{name: -1}) == INVALID
    assert keep(p, max_keep=0) == INVALID and evict(p, max_keep=0) == INVALID
    assert keep(p, max_keep=(1 << 30) + 1) == evict(p, max_keep=(1 << 30) + 1) == UNSUPPORTED
    assert keep(params(batch=65536, n_q_heads=1024, n_kv_heads=1024)) == UNSUPPORTED
    # (more tiles than are counted in 31 bits)
    assert weigh(params(batch=65536, max_pages=1 << 20, n_q_heads=64, n_kv_heads=64)) == UNSUPPORTED


def test_workspace():
    long = params(max_pages=4000)                             # 64000 keys of six heads: several workgroups to a head
    need = mp.magicpig_paged_workspace_bytes(long)
    assert keep(long, workspace=None) == SMALL and keep(long, bytes=4096) == SMALL
    assert need >= 6 * 8 * 12 * 1024


@accepted
def test_what_is_accepted_gets_as_far_as_the_launch():
    for p in (params(), params(max_pages=4000), params(dtype="fp32"), params(kv_dtype="fp8"), params(max_new=1 << 24)):
        assert [call(p) for call in CALLS] == [LAUNCH] * 3
    assert keep(params(), workspace=None, bytes=0) == LAUNCH
    long = params(max_pages=4000)
    assert keep(long, bytes=mp.magicpig_paged_workspace_bytes(long)) == LAUNCH
    four = params(kv_dtype="mxfp4")
    assert weigh(four, k_block_scales=FAKE) == evict(four, k_block_scales=FAKE, v_block_scales=FAKE) == LAUNCH
    assert weigh(params(kv_dtype="fp8"), k_scale=FAKE, counted=None, token_start=None) == LAUNCH
    assert evict(params(), kept=None, max_keep=0, weights=None) == LAUNCH
    assert weigh(params(batch=0)) == keep(params(batch=0)) == OK
    assert weigh(params(q_strides=(1 << 22, 1 << 22))) == LAUNCH


def arguments(p):
    bf, f32 = torch.bfloat16, torch.float32
    pool, weights = posing(p.n_pages, 16, 2, 128, dtype=bf), posing(p.n_pages, 2, 16, dtype=f32)
    i = posing(3)
    return {"weigh": dict(q=posing(p.max_tokens, 8, 128, dtype=bf), k_pages=pool, k_scale=None, k_block_scales=None, block_table=posing(3, p.max_pages),
                          lengths=i, token_start=posing(4), lse=posing(p.max_tokens, 8, dtype=f32), counted=i, weights=weights),
            "keep": dict(weights=weights, block_table=posing(3, p.max_pages), lengths=i, budgets=i, n_first=1, n_last=2, kept=posing(3, 2, 50), lengths_out=i),
            "evict": dict(kept=posing(3, 2, 50), lengths=i, lengths_kept=i, block_table=posing(3, p.max_pages), free_pages=posing(p.n_pages), n_free=posing(1),
                          k_pages=pool, v_pages=pool, k_block_scales=None, v_block_scales=None, weights=weights, n_free_out=posing(1), status=posing(1))}


BOUND = {"weigh": mp.magicpig_page_weights, "keep": mp.magicpig_page_keep, "evict": mp.magicpig_page_evict}


@pytest.mark.parametrize("which,name,tensor", [
    ("weigh", "q", lambda: posing(12, 8, 128)), ("weigh", "k_pages", lambda: posing(99, 16, 2, 128, dtype=torch.bfloat16)),
    ("weigh", "lse", lambda: posing(12, 7, dtype=torch.float32)), ("weigh", "lse", lambda: None), ("weigh", "counted", lambda: posing(2)),
    ("weigh", "weights", lambda: posing(100, 2, 16)), ("weigh", "k_block_scales", lambda: posing(100, 16, 2, 4, dtype=torch.uint8)),
    ("weigh", "lengths", lambda: posing(3, device=1)), ("keep", "weights", lambda: posing(100, 2, 15, dtype=torch.float32)),
    ("keep", "budgets", lambda: None), ("keep", "kept", lambda: posing(3, 1, 50)), ("keep", "kept", lambda: None), ("keep", "lengths_out", lambda: posing(3, dtype=torch.int64)),
    ("evict", "kept", lambda: posing(2, 2, 50)), ("evict", "free_pages", lambda: posing(99)), ("evict", "status", lambda: None),
    ("evict", "v_pages", lambda: posing(100, 16, 2, 127, dtype=torch.bfloat16)), ("evict", "weights", lambda: posing(100, 2, 15, dtype=torch.float32)),
    ("evict", "v_block_scales", lambda: posing(100, 16, 2, 4, dtype=torch.uint8)), ("evict", "lengths_kept", lambda: posing(2))])
def test_binding_refuses_tensors_that_do_not_fit(which, name, tensor):
    p = params()
    got = arguments(p)[which]
    got[name] = tensor()
    with pytest.raises(mp.MagicpigError, match=name if not isinstance(got[name], torch.Tensor) or got[name].get_device() == 0 else "device"):
        BOUND[which](p, **got)


def test_binding_passes_on_what_fits(monkeypatch):
    calls = []
    monkeypatch.setattr(mp, "_paged_call", lambda *a: calls.append(a))
    p = params()
    for which, got in arguments(p).items():
        BOUND[which](p, **got)
    without = arguments(p)["evict"]
    without.update(kept=None, weights=None)
    mp.magicpig_page_evict(p, **without)
    assert len(calls) == 4 and all(a[2]._obj is p for a in calls)
    assert calls[1][8] == 2 and calls[1][9] == 50 and calls[3][3:5] == (None, 0)
    for name in ("k_block_scales", "v_block_scales"):         # block scales that are missing
        with pytest.raises(mp.MagicpigError, match="k_block_scales|k_pages"):
            BOUND["evict"](params(kv_dtype="mxfp4"), **arguments(p)["evict"])
