"""Every kernel and configuration of the log probability and embedding calls at a size that takes it: which kernels were launched.  (Their results at such
sizes: test_gpu_logprobs.py, test_gpu_embed.py, and below where a line of the dispatch is met by no size there.)"""
import pytest
import torch

from test_gpu_logprobs import check_forward, check_gradients, rows, some_tokens
from test_gpu_operator_routes import launched

pytestmark = pytest.mark.gpu
PART, FINISH, GRAD, ROW, TOP, MERGE = ("logprob_part_kernel", "logprob_finish_kernel", "logprob_grad_kernel", "logprob_row_kernel", "topk_part_kernel",
                                       "topk_merge_kernel")


@pytest.mark.parametrize("kind,B,N,k,kernels", [
    ("bf16", 8, 128256, 0, [PART, FINISH]), ("bf16", 127, 70000, 0, [PART, FINISH]), ("bf16", 600, 40000, 0, [PART]), ("bf16", 1024, 40000, 0, [PART]),
    ("bf16", 3, 4096, 0, [ROW]), ("bf16", 3, 4097, 0, [ROW]), ("bf16", 3, 8193, 0, [ROW]), ("bf16", 3, 16385, 0, [ROW]), ("bf16", 3, 32769, 0, [ROW]),
    ("bf16", 256, 65536, 0, [ROW]), ("bf16", 257, 65536, 0, [PART, FINISH]), ("bf16", 3, 65537, 0, [PART, FINISH]),
    ("f32", 300, 2049, 0, [ROW]), ("f32", 600, 4097, 0, [ROW]), ("f32", 512, 16384, 0, [ROW]), ("f32", 257, 16385, 0, [PART, FINISH]), ("f32", 33, 32768, 0, [ROW]),
    ("prob", 512, 9000, 0, [ROW]), ("prob", 513, 9000, 0, [PART]), ("prob", 600, 8192, 0, [ROW]), ("prob", 256, 32768, 0, [ROW]), ("prob", 9, 32769, 0, [PART, FINISH]),
    ("bf16", 8, 128256, 5, [TOP, MERGE]), ("bf16", 200, 5000, 5, [TOP]), ("prob", 4, 30000, 128, [TOP, MERGE]),
])
def test_forward(kind, B, N, k, kernels):
    from paper_2506_03206_amd import rdk
    x, gen = rows(kind, B, N, B + N)
    tokens = some_tokens(B, N, 2, gen)
    o = rdk.LogprobsOutputs(B, 2, k, "cuda")
    assert launched([PART, FINISH, ROW, TOP, MERGE], lambda: rdk.rdk_logprobs(x, tokens, "prob" if kind == "prob" else "logit", k=k, outputs=o)) == kernels
    check_forward(x, tokens, kind, k=k)


def test_few_rows_of_many_tokens():
    """Rows for one workgroup of 1024 threads each, or spread over several where they are few and have more than two tokens."""
    from paper_2506_03206_amd import rdk
    for kind, B, C, kernels in (("bf16", 31, 3, [PART, FINISH]), ("bf16", 32, 3, [ROW]), ("bf16", 31, 2, [ROW]), ("prob", 32, 16, [ROW]), ("prob", 5, 3, [PART, FINISH])):
        x, gen = rows(kind, B, 32768 if kind == "prob" else 65536, B)
        tokens = some_tokens(B, x.shape[1], C, gen)
        assert launched([PART, FINISH, ROW], lambda: rdk.rdk_logprobs(x, tokens, "prob" if kind == "prob" else "logit")) == kernels
        check_forward(x, tokens, kind)


@pytest.mark.parametrize("kind,B,N,kernels", [
    ("bf16", 4, 4096, [ROW]), ("bf16", 300, 16385, [ROW]), ("f32", 4, 16384, [ROW]), ("f32", 4, 16385, [GRAD, ROW]), ("f32", 129, 16385, [ROW]),
    ("bf16", 127, 32769, [GRAD, ROW]), ("bf16", 128, 32769, [ROW]), ("bf16", 129, 131072, [ROW]), ("bf16", 129, 131073, [PART, FINISH, GRAD]),
    ("f32", 600, 65537, [PART, GRAD]), ("bf16", 100, 65537, [PART, FINISH, GRAD]),
])
def test_step(kind, B, N, kernels):
    from paper_2506_03206_amd import rdk
    x, gen = rows(kind, B, N, B + N)
    tokens, g = some_tokens(B, N, 1, gen), torch.randn((B, 1), generator=gen, device="cuda")
    o = rdk.LogprobsOutputs(B, 1, 0, "cuda", grad=torch.empty_like(x))
    assert launched([PART, FINISH, GRAD, ROW], lambda: rdk.rdk_logprobs_step(x, tokens, g, outputs=o)) == kernels
    check_gradients(x, tokens, kind, 1.0, g, torch.randn(B, generator=gen, device="cuda"))


@pytest.mark.parametrize("B,accumulate,kernels", [
    (1024, False, ["embed_grad_few_kernel"]), (1025, False, ["embed_sort_kernel", "embed_grad_sum_kernel", "embed_grad_join_kernel"]),
    (20480, True, ["embed_sort_kernel", "embed_grad_sum_kernel", "embed_grad_join_kernel"]),
    (20481, True, ["embed_count_kernel", "embed_scan_kernel", "embed_place_kernel", "embed_grad_sum_kernel", "embed_grad_join_kernel"]),
])
def test_embedding(B, accumulate, kernels):
    from paper_2506_03206_amd import rdk
    names = ["embed_kernel", "embed_grad_few_kernel", "embed_sort_kernel", "embed_count_kernel", "embed_scan_kernel", "embed_place_kernel",
             "embed_grad_sum_kernel", "embed_grad_join_kernel"]
    ids = torch.randint(0, 500, (B,), device="cuda", dtype=torch.int32)
    o = rdk.EmbedGradOutputs(500, 16, torch.float32, "cuda", grad=torch.zeros((500, 16), device="cuda"))
    assert launched(names, lambda: rdk.rdk_embed_grad(ids, torch.ones((B, 16), device="cuda"), o, accumulate=accumulate)) == kernels
    assert torch.equal(o.grad[:, 3], torch.bincount(ids.long(), minlength=500).float())
    assert launched(names, lambda: rdk.rdk_embed(ids, o.grad)) == ["embed_kernel"]


def test_more_tokens_than_small_tiles_hold():
    """Tiles of four times as many tokens, from 524289 on."""
    from test_gpu_embed import check_gradient, generator, tokens
    gen = generator(1)
    ids = tokens("zipf", 524289 + 3000, 400000, gen)
    check_gradient(ids, torch.randn((ids.numel(), 4), generator=gen, device="cuda"), 400000, torch.float32, 1.0, False)
