"""Which keys stay where the lengths that are left are written over those that are read."""
import numpy as np
import pytest
import torch

from paper_2410_16179_amd import binding as mp
from tests import evict_reference as ev
from tests.test_gpu_page_keep import problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("over", ["lengths", "budgets"])
# one workgroup to a KV head, small and large, and several
@pytest.mark.parametrize("lengths,kv_heads", [([300, 0, 17, 5000, 40], 8), (list(range(0, 900, 3)), 4), ([20000, 300], 8), ([70000, 12, 33000], 4)])
def test_every_head_sees_the_same_lengths(over, lengths, kv_heads):
    rng = np.random.default_rng(kv_heads)
    table, w = problem(rng, lengths, kv_heads, 16)
    budgets = [int(x) for x in rng.integers(-1, 300, len(lengths))]
    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()
    p = mp.make_paged_params(batch=len(lengths), n_q_heads=kv_heads, n_kv_heads=kv_heads, dtype="bf16", page_size=16, max_pages=table.shape[1],
                             n_pages=w.shape[0])
    ws, accounts, dtable = mp.alloc_paged_workspace(p), torch.from_numpy(w).cuda(), i32(table)
    want, want_out = ev.keep(w, table, lengths, budgets, 2, 5, 250)
    graph = torch.cuda.CUDAGraph()
    at = {"lengths": i32(lengths), "budgets": i32(budgets)}
    kept = torch.full((len(lengths), kv_heads, 250), 12345, dtype=torch.int32, device="cuda")
    call = lambda: mp.magicpig_page_keep(p, accounts, dtable, at["lengths"], at["budgets"], 2, 5, kept, at[over], ws)
    call()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    for run in [call, graph.replay, graph.replay]:
        at["lengths"].copy_(i32(lengths))
        at["budgets"].copy_(i32(budgets))
        kept.fill_(12345)
        run()
        np.testing.assert_array_equal(at[over].cpu().numpy(), want_out)
        np.testing.assert_array_equal(kept.cpu().numpy(), want)
