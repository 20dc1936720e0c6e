"""The K best of rows that are still longer than one workgroup holds after they have
been shortened: whole rows against a stable sort, on the GPU."""
import pytest
import torch

from paper_2606_01502_amd import mla

pytestmark = pytest.mark.gpu


def rows(N, K, how, shape=(2, 1)):
    g = torch.Generator(device="cuda").manual_seed(N + K)
    x = torch.rand((*shape, N), generator=g, device="cuda")
    if how == "ties":
        x = torch.round(x * 30)
    if how == "holes":
        x[0, 0, : N // 2] = -float("inf")
        x[1, 0, 100:] = -float("inf")  # (fewer than K)
    return x


def best(x, K):
    """Of equal ones the first, never -inf, places rising, -1 behind the last."""
    N = x.shape[-1]
    v, at = torch.sort(x, dim=-1, descending=True, stable=True)
    at = torch.where(v[..., :K] == -float("inf"), N, at[..., :K])
    want = torch.sort(at, dim=-1).values
    return torch.where(want == N, -1, want)


# The K best of each 8192 make up the shorter row.  After one step (the first five) and
# after two (the sixth) these still hold over 65,536 values, and another step would not
# halve them.  Of 131,072 values with K 4096 a step leaves 65,536; with one value or pick
# more there is no first step.
@pytest.mark.parametrize("N,K", [(139264, 4096), (131137, 3856), (150000, 3900), (200000, 4000), (827392, 4090),
                                 (278528, 4096), (131072, 4096), (131073, 4096), (131072, 4097)])
@pytest.mark.parametrize("how", ["random", "ties", "holes"])
def test_topk_of_rows_that_stay_long(N, K, how):
    print(f"case: topk {N} {K} {how}", flush=True)
    x = rows(N, K, how)
    assert torch.equal(mla.select_topk(x, K).long(), best(x, K))


@pytest.mark.parametrize("K", [3856, 3900, 4000, 4095, 4096, 4097, 8192])
def test_topk_of_random_lengths(K):
    g = torch.Generator().manual_seed(K)
    for N in torch.randint(65537, 1 << 20, (6,), generator=g).tolist():
        print(f"case: topk {N} {K}", flush=True)
        x = rows(N, K, "random", (1, 3))
        assert torch.equal(mla.select_topk(x, K).long(), best(x, K)), N


def test_topk_of_rows_that_stay_long_strided():
    """Rows apart by more than they hold, scores and ids."""
    N, K = 155000, 3950
    wide = torch.rand((2, 4, N + 77), device="cuda")
    ids = torch.full((2, 4, K + 9), 5, dtype=torch.int32, device="cuda")
    x = wide[:, ::2, 33:33 + N]
    mla.select_topk(x, ids=ids[:, ::2, 4:4 + K])
    assert torch.equal(ids[:, ::2, 4:4 + K].long(), best(x, K))
    assert (ids[:, 1::2] == 5).all() and (ids[..., :4] == 5).all() and (ids[..., 4 + K:] == 5).all()
