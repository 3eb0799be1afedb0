"""Rows to and from pools in four bits, byte for byte."""
import numpy as np
import pytest
import torch

from paper_2410_16179_amd import binding as mp
from tests import mxfp_reference as mx

pytestmark = pytest.mark.gpu
D = 128


def pools(n_pages, page, heads, layout, fill=0xa5):
    """Two pools and their block scales, views in (page, key, head) order, with room for wider rows."""
    def one(width):
        wide = width * (2 if layout == "wide" else 1)
        if layout == "head":
            return torch.full((n_pages, heads, page, width), fill, dtype=torch.uint8, device="cuda").permute(0, 2, 1, 3)
        return torch.full((n_pages, page, heads, wide), fill, dtype=torch.uint8, device="cuda")[..., :width]
    return one(64), one(64), one(4), one(4)


def params(k, tokens, rows, **more):
    n_pages, page, heads, _ = k.shape
    s = tuple(2 * x for x in k.stride()[:3])
    return mp.make_paged_params(**{**dict(batch=1, n_q_heads=heads, n_kv_heads=heads, dtype="bf16", kv_dtype="mxfp4", page_size=page, max_pages=n_pages,
                                          n_pages=n_pages, max_tokens=tokens, max_new=tokens, k_strides=s, v_strides=s,
                                          k_new_strides=rows.stride()[:2], v_new_strides=rows.stride()[:2]), **more})


def special_rows(rng, tokens, heads):
    """Rows of many sizes, zeros, borders of the rounding, values at both ends of bf16, infinities and NaN."""
    x = rng.standard_normal((tokens, heads, 4, 32)) * 2.0 ** rng.integers(-130, 126, (tokens, heads, 4, 1))
    if tokens > 6:
        x[0] = 0.0
        x[1, :, 0] = np.tile([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], 4)
        x[1, :, 1] = -np.tile([0.2490234375, 0.7490234375, 1.2578125, 1.7421875, 2.515625, 3.484375, 5.03125, 6.03125], 4)
        x[2, :, 2] = 3.3895313892515355e38 * np.linspace(-1, 1, 32)
        x[3, :, 1, 5], x[3, :, 2, 31], x[3, :, 3, 0] = np.nan, np.inf, -np.inf
        x[4] = rng.integers(-40, 40, (heads, 4, 32)) * 2.0 ** -133
        x[5, :, 3] = -0.0
    return torch.from_numpy(x.reshape(tokens, heads, D)).float().to(torch.bfloat16)


@pytest.mark.parametrize("tokens,heads,page", [(1, 1, 16), (7, 3, 16), (64, 8, 64), (333, 2, 1024), (3001, 8, 32)])
@pytest.mark.parametrize("layout", ["token", "head", "wide"])
def test_append_and_read(tokens, heads, page, layout):
    rng = np.random.default_rng(tokens)
    n_pages = -(-tokens // page) + 2
    kp, vp, kb, vb = pools(n_pages, page, heads, layout)
    before = [t.clone() for t in (kp, vp, kb, vb)]
    rows = [special_rows(rng, tokens, 2 * heads).cuda() for _ in range(2)]
    k, v = rows[0][:, :heads], rows[1][:, heads:]             # (strided: from one product)
    slots = torch.from_numpy(rng.permutation(n_pages * page)[:tokens]).cuda()
    if tokens > 6:
        slots[[5, 6]] = torch.tensor([-1, n_pages * page], device="cuda")
        slots[tokens - 1] = -2 ** 62
    p = params(kp, tokens, k)
    mp.magicpig_page_append_mxfp(p, k, v, slots, kp, vp, kb, vb)
    at = slots.cpu().numpy()
    real = (at >= 0) & (at < n_pages * page)
    for pool, block, old, old_block, new in ((kp, kb, before[0], before[2], k), (vp, vb, before[1], before[3], v)):
        want_rows, want_scales = mx.quantise(new.cpu().double().numpy())
        # the bytes of a block that is NaN stand for nothing
        alive = np.repeat(want_scales != 255, 16, -1)
        want, want_block = old.cpu().numpy().copy(), old_block.cpu().numpy().copy()
        got, got_block = pool.cpu().numpy(), block.cpu().numpy()
        for t in np.nonzero(real)[0]:
            pg, i = at[t] // page, at[t] % page
            want[pg, i] = np.where(alive[t], want_rows[t], got[pg, i])
            want_block[pg, i] = want_scales[t]
        np.testing.assert_array_equal(got, want)
        np.testing.assert_array_equal(got_block, want_block)
    # back again; rows without a slot stay as they are
    out = torch.full((tokens, 2 * heads + 1, D), 7.0, dtype=torch.bfloat16, device="cuda")
    ko, vo = out[:, :heads], out[:, heads:2 * heads]
    mp.magicpig_page_read_mxfp(params(kp, tokens, ko), kp, vp, kb, vb, slots, ko, vo)
    for new, got in ((k, ko), (v, vo)):
        want = mx.values(*mx.quantise(new.cpu().double().numpy()))
        got = got.cpu().double().numpy()
        np.testing.assert_array_equal(got[real], want[real])
        np.testing.assert_array_equal(got[~real], 7.0)
    assert (out[:, 2 * heads] == 7.0).all()


def test_every_byte_and_scale_reads_as_what_it_stands_for():
    page, heads = 16, 1
    kp, vp, kb, vb = pools(16, page, heads, "token")
    rng = np.random.default_rng(3)
    for pool in (kp, vp):
        pool.copy_(torch.from_numpy(rng.integers(0, 256, pool.shape).astype(np.uint8)))
    kb.copy_(torch.arange(1024, dtype=torch.int32).remainder(256).to(torch.uint8).reshape(kb.shape))
    vb.copy_(255 - kb)
    slots = torch.arange(256, device="cuda")
    ko, vo = (torch.zeros(256, heads, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mp.magicpig_page_read_mxfp(params(kp, 256, ko), kp, vp, kb, vb, slots, ko, vo)
    for pool, block, got in ((kp, kb, ko), (vp, vb, vo)):
        with np.errstate(over="ignore"):
            want = mx.values(pool.cpu().numpy().reshape(256, 1, 64), block.cpu().numpy().reshape(256, 1, 4)).astype(np.float32)
        np.testing.assert_array_equal(got.float().cpu().numpy(), want)


def test_far_pools():
    page, heads = 16, 1
    n_pages = (9 << 30) // 64 // page                         # pools beyond 8 GiB, block scales beyond 512 MiB
    kp, vp = (torch.empty(n_pages, page, heads, 64, dtype=torch.uint8, device="cuda") for _ in range(2))
    kb, vb = (torch.empty(n_pages, page, heads, 4, dtype=torch.uint8, device="cuda") for _ in range(2))
    x = special_rows(np.random.default_rng(5), 3, heads).cuda()
    slots = torch.tensor([n_pages * page - 1, n_pages * page // 2 + 3, 5], device="cuda")
    p = params(kp, 3, x)
    mp.magicpig_page_append_mxfp(p, x, -x, slots, kp, vp, kb, vb)
    ko, vo = torch.zeros_like(x), torch.zeros_like(x)
    mp.magicpig_page_read_mxfp(p, kp, vp, kb, vb, slots, ko, vo)
    want = mx.values(*mx.quantise(x.cpu().double().numpy()))
    np.testing.assert_array_equal(ko.cpu().double().numpy(), want)
    np.testing.assert_array_equal(vo.cpu().double().numpy(), -want)
