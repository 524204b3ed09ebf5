"""The choice of pages where more scores than a few are next to the border, in tables that several warps of a CTA share: how many counts a list takes before
its exact scores are counted hangs on the scores, so tokens of every number of them stand side by side, again and again."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [257, 1000, 1025, 2048, 2100, 5000, 17000])    # four warps, eight, up to 8, 32 and 64 pages a lane, any number
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_more_close_scores_than_are_looked_at_one_by_one(n, dtype):
    from paper_2311_00368_b200 import binding as b
    M, Hkv, d = 40, 2, 8
    pages = M * n
    means = b.paged_means(pages, Hkv, d, dtype)
    rng = np.random.default_rng(n)
    score = np.full((M, n, Hkv), 1.0)
    for i in range(M):   # all alike but a few better ones, further and further away: more and more halvings, each a count
        score[i, rng.permutation(n)[:1 + i % 3], 0] = 1 + 2.0 ** (i % 20 - 7)
        score[i, rng.permutation(n)[:i % 2], 1] = 2.0 ** (i - 20) + 1
    means[..., 0] = torch.from_numpy(score.reshape(pages, Hkv)).to(dtype).cuda()
    score = means[..., 0].cpu().double().numpy().reshape(M, n, Hkv)
    q = torch.zeros((M, Hkv, d), dtype=dtype, device="cuda")
    q[..., 0] = 1
    tables = torch.arange(pages, dtype=torch.int32, device="cuda").view(M, n)
    seen = torch.full((M,), n, dtype=torch.int32, device="cuda")
    for keep, first, last in ((9, 0, 0), (33, 1, 2), (120, 0, 1), (n - 2, 1, 1)):
        want = np.empty((M, Hkv, keep), np.int32)
        for i in range(M):
            for g in range(Hkv):
                y = score[i, :, g].copy()
                y[:first] = y[n - last:] = np.inf
                want[i, g] = np.sort(np.lexsort((np.arange(n), -y))[:keep])
        want = torch.from_numpy(want).cuda()
        for _ in range(25):
            assert torch.equal(b.paged_select(q, means, tables, seen, 1, keep, first, last, dtype=dtype), want)
