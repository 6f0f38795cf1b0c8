"""What cfgzip_head_loss_grad keeps in its workspace, without a GPU: pieces of the vocabulary hold dz and, of bf16 rows, the weights in
fp16 beside it."""

import os

import pytest

MB = 1 << 20


@pytest.fixture(scope="module")
def need():
    from paper_2605_29986_amd import binding, build
    if not os.path.exists(binding.library_path()):
        build.build()
    lib = binding.load_library()
    return lambda N, V, D: lib.cfgzip_head_loss_grad_workspace_bytes(N, V, D, 2)


@pytest.mark.parametrize("N,V,D", [(257, 128256, 4096), (300, 128256, 4096), (1000, 128256, 4096), (4096, 128256, 4096), (2048, 151936, 2048),
                                   (200, 151936, 4001)])
def test_pieces_of_many_rows(need, N, V, D):
    """224 MB of dz and fp16 weights, three times as much where rows times hidden size are few (2e11 products of a token and a row for a
    piece), or the tokens of 256 tiles of 256 x 256 or 256 x 128 if those are more; beside them two copies of
    the hidden states in 16 bits and one in 32 for each share of the sum (shares' tiles of 256 x 128 go up to two rounds of 256)."""
    rows, d = (N + 255) // 256 * 256, (D + 63) // 64 * 64
    tokens = 256 // (rows // 256) * 256
    piece = max(224 * MB, min(3 * 224 * MB, (2e11 / N / D + tokens) * 2 * (rows + d)), 2 * tokens * (rows + d), 2048 * 2 * (rows + d))
    shares = max(1, 512 // ((D + 255) // 256 * ((N + 127) // 128)))
    assert need(N, V, D) < piece + rows * d * (4 + 4 * shares) + 2 * MB


def test_pieces_do_not_grow_with_the_vocabulary(need):
    """Behind one piece nothing grows but the tokens' masks, of which there are none here, and of fp16 rows which token is whose target:
    eight bytes a token."""
    assert need(4096, 4_000_000, 4096) <= need(4096, 128256, 4096) + 8 * (4_000_000 - 128256) + MB


@pytest.mark.parametrize("N", [1, 16, 128, 256])
def test_few_rows_keep_their_logits(need, N):
    """Logits in 32 bits and dz in twice 16 of every token, and no copy of the weights."""
    V, D = 128256, 4096
    rows = max(2 * N, 64)
    assert need(N, V, D) < (N * 4 + rows * 2) * (V + 256) + 2 * N * D * 4 * 64 + 4 * MB
