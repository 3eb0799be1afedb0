"""The sizes that the calls on accounts take and refuse, on both sides of the borders."""
import ctypes

import pytest

from paper_2410_16179_amd import binding as mp
from tests.test_evict_host import keep, weigh
from tests.test_paged_host import FAKE, LAUNCH, UNSUPPORTED, accepted, params
from tests.test_smaller_cache_plan import plan, weights  # noqa: F401  (a fixture, and what it is called by)

# keys of a tile in each form: (bits of a key's element, query heads a KV head, new tokens) -> the smallest there is
FORMS = {(16, 4, 1): 32, (8, 4, 1): 64, (4, 4, 1): 64, (8, 8, 4): 32, (4, 64, 2): 32, (16, 64, 64): 64, (8, 64, 64): 64, (4, 64, 64): 64, (32, 4, 1): 16, (32, 64, 64): 32}


@pytest.mark.parametrize("bits,group,new", list(FORMS))
# (requests, KV heads, keys): 2^35 of them, long requests and many, and one page more than a tile goes into
@pytest.mark.parametrize("batch,kv,keys", [(32, 1, 1 << 30), (4, 8, 1 << 30), (65536, 1, 1 << 19), (65536, 1024, 512), (65536, 1024, 496), (63 * 1024, 1024, 16 * 32), (4096, 8, (1 << 20) - 16)])
def test_what_is_said_to_be_taken_is(plan, bits, group, new, batch, kv, keys):  # noqa: F811
    if bits == 32:
        batch //= 2
    assert batch * kv * keys <= 1 << (34 if bits == 32 else 35)
    assert weights(plan, batch, kv, group, new, keys, fp32=bits == 32, bits=min(bits, 16))["fit"]


@pytest.mark.parametrize("bits,group,new", list(FORMS))
def test_the_border_is_where_tiles_are_no_longer_counted(plan, bits, group, new):  # noqa: F811
    form = lambda batch: weights(plan, batch, 8, group, new, 1 << 26, fp32=bits == 32, bits=min(bits, 16))
    per = form(1)["tiles"]                                    # of a request, with the tile of long tables
    assert per % (8 << 18) == 0 and per <= (8 << 26) // FORMS[bits, group, new]
    first = (2 ** 31 - 1024) // per                           # requests whose tiles are counted
    assert form(first)["fit"] and not form(first + 1)["fit"]


def problem(pages, **kw):
    return params(batch=65536, n_q_heads=64, n_kv_heads=64, max_pages=pages, max_tokens=65536, max_new=1, **kw)


def test_larger_ones_are_refused():
    # 2^22 requests times KV heads: tiles of 32 keys (bf16), of 64 (fewer bits), of 16 (float32)
    # (1023 pages of 16 keys are 511 tiles and a half)
    assert weigh(problem(1024)) == weigh(problem(1023)) == UNSUPPORTED
    assert weigh(problem(2048, kv_dtype="fp8")) == weigh(problem(2048, kv_dtype="mxfp4"), k_block_scales=FAKE) == UNSUPPORTED
    assert weigh(problem(512, dtype="fp32")) == UNSUPPORTED
    assert keep(problem(1)) == UNSUPPORTED


@accepted
def test_and_smaller_ones_get_as_far_as_the_launch():
    assert weigh(problem(512)) == weigh(problem(1022)) == LAUNCH
    assert weigh(problem(1024, kv_dtype="fp8")) == weigh(problem(1024, kv_dtype="mxfp4"), k_block_scales=FAKE) == LAUNCH
    assert weigh(problem(256, dtype="fp32")) == weigh(problem(511, dtype="fp32")) == LAUNCH
    fewer = problem(1)
    fewer.n_kv_heads = fewer.n_q_heads = 63
    assert keep(fewer) == LAUNCH
    assert mp.lib().magicpig_paged_workspace_bytes(ctypes.byref(fewer)) > 0
