"""The table's gradient of batches whose sorted tokens are cut into pieces of 32 (from 65536 groups of 64 threads on: 17000 tokens of 1024 fp32 columns, 2048 bf16): runs of
equal tokens that begin and end in every position around a piece's end, and runs over more pieces than a wavefront looks ahead.

Rows are whole numbers up to 8 and sums stay below 2^24, so that every sum is exact in any order, and a bf16 result is the exact one rounded."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def data():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(21)
    return gen, torch.randint(-8, 9, (17400, 2048), generator=gen, device="cuda").float()


def check(ids, rows, V, table, accumulate):
    from paper_2506_03206_amd import rdk
    B, d = rows.shape
    held = (ids >= 0) & (ids < V)
    which = (torch.arange(V, device="cuda")[:, None] == torch.where(held, ids, -1)[None, :]).double()
    want = which @ rows.double()
    old = torch.full((V, d), 3.0, device="cuda").to(table)
    o = rdk.EmbedGradOutputs(V, d, table, "cuda", grad=old.clone() if accumulate else torch.full((V, d), float("nan"), device="cuda").to(table))
    rdk.rdk_embed_grad(ids, rows, o, 0.5, None, accumulate)
    want = want * 0.5 + (3.0 if accumulate else 0.0)
    assert float(want.abs().max()) < 2 ** 24
    if accumulate:                                                      # rows without tokens are left
        want[which.sum(1) == 0] = 3.0
    assert torch.equal(o.grad, want.to(table))


@pytest.mark.parametrize("table,rows", [(F32, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("first", [0, 1, 31, 32, 33])
def test_runs_around_the_ends_of_pieces(data, table, rows, first):
    """Tokens 0, 1, 2 in runs of `first`, `length` and the rest, in any order in the batch."""
    gen, x = data
    d = 2048 if (table, rows) == (BF16, BF16) else 1024
    for length in (1, 31, 32, 33, 64, 65, 2100):
        ids = torch.cat([torch.zeros(first), torch.ones(length), torch.full((17000 - length,), 2.0), torch.arange(3, 60)]).to(torch.int32).cuda()
        ids = ids[torch.randperm(ids.numel(), generator=gen, device="cuda")]
        check(ids, x[: ids.numel(), :d].contiguous().to(rows), 64, table, length % 2 == 0)


@pytest.mark.parametrize("table,rows", [(F32, F32), (BF16, BF16)])
def test_short_and_long_runs(data, table, rows):
    """One run over all 544 pieces; runs of 1 to 70 tokens one behind the other; unknown ids behind them, in whole pieces too."""
    gen, x = data
    d = 2048 if table == BF16 else 1024
    x = x[:17400, :d].contiguous().to(rows)
    check(torch.full((17400,), 5, dtype=torch.int32, device="cuda"), x, 7, table, False)
    lengths = torch.randint(1, 71, (1000,), generator=gen, device="cuda")
    ids = torch.repeat_interleave(torch.arange(1000, device="cuda"), lengths)[:17400].to(torch.int32)
    assert ids.numel() == 17400
    ids = ids[torch.randperm(17400, generator=gen, device="cuda")]
    for unknown in (0, 1, 40, 5000):
        ids[:unknown] = torch.where(torch.arange(unknown, device="cuda") % 2 == 0, -1, 1000).to(torch.int32)
        check(ids, x, 1000, table, unknown == 40)
