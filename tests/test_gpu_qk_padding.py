"""Head norms with padding rows (an index outside the table) whose outputs the call makes itself: those rows come out as
zeros, whatever the memory held before."""
import pytest
import torch

from paper_2607_12287_amd import incvit
from tests.test_gpu_qk import make, make_table

pytestmark = pytest.mark.gpu


def leave_nan_behind(*tensors):
    """Blocks of these sizes that hold NaN go back to the allocator, which hands them out again."""
    old = [torch.full_like(t, float("nan")) for t in tensors]
    torch.cuda.synchronize()
    del old


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,hq,hk,d", [(9, 4, 2, 64), (300, 16, 16, 72)])
def test_padding_rows_of_outputs_that_the_call_makes(dtype, rows, hq, hk, d):
    q, k, qg, kg, _, _ = make(rows, hq, hk, d, dtype)
    table = make_table(rows, d // 2)
    index = torch.arange(rows, dtype=torch.int32, device="cuda")
    index[1::3] = -1
    index[2] = rows
    live = (index >= 0) & (index < rows)
    want_q, want_k = incvit.qk_norm_rope(q, k, table, q_gamma=qg, k_gamma=kg)
    leave_nan_behind(q, k)
    qo, ko = incvit.qk_norm_rope(q, k, table, q_gamma=qg, k_gamma=kg, index=index)
    for got, want in ((qo, want_q), (ko, want_k)):
        assert torch.equal(got[live], want[live])
        assert torch.equal(got[~live], torch.zeros_like(got[~live]))


def test_without_a_rotation_the_index_is_not_looked_at():
    q, k, qg, kg, _, _ = make(7, 4, 2, 64, "bf16")
    index = torch.full((7,), -1, dtype=torch.int32, device="cuda")
    for a, b in zip(incvit.qk_norm_rope(q, k, q_gamma=qg, k_gamma=kg, index=index), incvit.qk_norm_rope(q, k, q_gamma=qg, k_gamma=kg)):
        assert torch.equal(a, b)


def test_captured_and_replayed():
    """New outputs inside a captured call: each replay starts them from zeros, whatever was written to them between."""
    q, k, qg, kg, _, _ = make(40, 16, 16, 72, "bf16")
    table = make_table(64, 36)
    index = torch.arange(40, dtype=torch.int32, device="cuda")
    run = lambda: incvit.qk_norm_rope(q, k, table, q_gamma=qg, k_gamma=kg, index=index)  # noqa: E731
    run()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = run()
    for seed in range(3):
        index.copy_(torch.randint(-30, 64, (40,), generator=torch.Generator().manual_seed(seed)))
        for t in out:
            t.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, run()):
            assert torch.equal(a, b) and not b[index < 0].any()
