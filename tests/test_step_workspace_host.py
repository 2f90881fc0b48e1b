"""Host-only: the workspaces of the table's gradient and of the backward norms have the sizes that the headers state, and not more."""
import pytest

from paper_2506_13996_amd import binding as B

MB = 1 << 20


@pytest.mark.parametrize("H", [8, 512, 520, 1600, 4096, 8192])
@pytest.mark.parametrize("V", [1, 50257, 128256])
def test_embedding_workspace(H, V):
    for N in (1, 7, 100, 3001, 4096, 4097, 16384, 65536, 131072, 300000, 1 << 20):
        # sums of cut tokens: two rows of fp32 for each range of 128 sorted rows, or of fewer where calls are short
        sums = max(N * H / 16, min(N * H, 32 * MB))
        # 16 bytes a row in sorted order, a mark a token; then 8 bytes a range (of 8 rows at least), 256 shares' counts, 256 bytes of
        # alignment and 8 rows of sums of a range that is begun for each term
        size = B.alst_embedding_workspace_bytes(N, H, V)
        assert 16 * N + V + N * H / 16 <= size <= 16 * N + V + sums + N + 256 * 512 * 4 + 8 * 256 + 8 * H, (N, H, V)


def test_block_norm_workspace():
    for H in (8, 504, 512, 520, 4096, 8192, 8200, 16384):
        most = 256 * 8 * H
        sizes = [B.alst_block_norm_workspace_bytes(N, H) for N in (1, 2, 255, 256, 257, 4096, 1 << 20, 1 << 30)]
        assert sizes == sorted(sizes) and sizes[0] == 8 * H and sizes[-1] == sizes[-2] == most
