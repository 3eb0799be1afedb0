"""Accounts of attention weight where a request's query rows lie far apart."""
import math

import numpy as np
import pytest
import torch

from paper_2410_16179_amd import binding as mp

pytestmark = pytest.mark.gpu
D, GROUP, KV, PAGE = 128, 43, 2, 64


@pytest.mark.parametrize("dtype,n", [("bf16", 1000), ("fp32", 520)])
def test_rows_of_one_request_beyond_two_gigabytes_of_offsets(dtype, n):
    # 43 heads a KV head: a step of rows ends inside a token, and tokens lie 2^22 elements apart, the largest stride
    rng, t = np.random.default_rng(n), torch.bfloat16 if dtype == "bf16" else torch.float32
    heads, pages = GROUP * KV, -(-n // PAGE)
    table = rng.permutation(pages + 2)[:pages]
    k = torch.from_numpy(rng.standard_normal((pages + 2, PAGE, KV, D))).to(t)
    q = torch.from_numpy(rng.standard_normal((n, heads, D))).to(t)
    keys, rows = k[table].reshape(-1, KV, D)[:n].double(), q.double()
    seen = torch.ones(n, n, dtype=torch.bool).tril()
    lse, want, off = torch.zeros(n, heads), torch.zeros(KV, n, dtype=torch.float64), torch.zeros(KV, n, dtype=torch.float64)
    for h in range(heads):
        g = h // GROUP
        x = rows[:, h] @ keys[:, g].T / math.sqrt(D)
        lse[:, h] = torch.logsumexp(x.masked_fill(~seen, -math.inf), -1).float()
        # how far float32 may be off: a score by 132 * 2^-24 of its products' magnitudes, the difference to lse by its rounding in base 2, the
        # exponential by two units
        l, reach = lse[:, h].double()[:, None], rows[:, h].abs() @ keys[:, g].abs().T / math.sqrt(D)
        w = torch.where(seen, torch.exp(x - l), 0.0)
        want[g] += w.sum(0)
        off[g] += (w * (132 * 2.0 ** -24 * reach + 2.0 ** -22 * (x.abs() + l.abs() + 2))).sum(0)
    off += (n * GROUP + 12) * 2.0 ** -24 * want
    p = dict(batch=1, n_q_heads=heads, n_kv_heads=KV, dtype=dtype, page_size=PAGE, max_pages=pages, n_pages=pages + 2, max_tokens=n, max_new=n)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    far = torch.empty((n - 1) * (1 << 22) + heads * D, dtype=t, device="cuda").as_strided((n, heads, D), (1 << 22, D, 1))
    far.copy_(q)
    got = []
    for x in (q.cuda(), far):
        accounts = torch.full((pages + 2, KV, PAGE), math.nan, device="cuda")
        mp.magicpig_page_weights(mp.make_paged_params(**p, q_strides=x.stride()[:2]), x, k.cuda(), None, None, i32(table[None]), i32([n]), i32([0, n]),
                                 lse.cuda(), None, accounts)
        got.append(accounts.cpu())
    assert torch.equal(got[0].view(torch.int32), got[1].view(torch.int32))
    w = got[0][table].double().permute(1, 0, 2).reshape(KV, -1)[:, :n]
    assert ((w - want).abs() <= off).all(), float(((w - want).abs() / off).max())
