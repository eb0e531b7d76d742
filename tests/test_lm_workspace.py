"""The vocabulary head's workspace against the account that the header gives of
it (CPU only: the queries read no memory)."""
import ctypes as ct

import pytest

from paper_1712_04048_amd import binding as B
from test_abi import _ensure_built

MB, SLACK = 1 << 20, 1 << 14   # of 24 buffers on boundaries of 256 bytes


def need(n, H, C, K, temp, bf, train):
    v = B.cavs_vocab(h_type=0, w_type=int(bf), n=n, H=H, C=C, label=16, K=K, alpha=0.5, temp=temp)
    return B.lib().cavs_vocab_workspace_bytes(ct.byref(v), int(train))


def up(x, m):
    return (x + m - 1) // m * m


def loss_bytes(n, H, C, K, temp, bf):
    """What the loss needs, but for the copy of W_s."""
    rows, words = up(n, 64 if n <= 64 else 256), up(C, 256)
    stat = 8 if not K else 12 if temp == 1.0 else 16
    return (rows * H * (2 if bf else 4) + rows * (words // (128 if bf else 64)) * stat
            + rows * (36 + (8 + 12 * K if K else 0)) + SLACK)


@pytest.mark.parametrize("bf", [False, True])
@pytest.mark.parametrize("K,temp", [(0, 1.0), (7, 1.0), (256, 2.0)])
@pytest.mark.parametrize("n,H,C", [
    (1, 64, 1), (64, 1024, 50001), (65, 64, 1 << 20), (300, 512, 10000), (4096, 1024, 32000),
    (8192, 2048, 128000), (32768, 64, 2048), (32769, 64, 2049), (65536, 1024, 100000),
    (65537, 512, 4097), (1 << 20, 64, 700), (1 << 20, 1024, 2048), (1 << 20, 1024, 2049),
    (1 << 20, 2112, 1 << 20), (1 << 20, 1 << 15, 1 << 20)])
def test_workspace_is_what_the_header_says(n, H, C, K, temp, bf):
    _ensure_built()
    e, rows = 2 if bf else 4, up(n, 64 if n <= 64 else 256)
    copy = H * up(C, 8) * 2 if bf and C % 8 else 0
    least = loss_bytes(n, H, C, K, temp, bf)
    got = need(n, H, C, K, temp, bf, False)
    assert least - 2 * SLACK <= got <= least + copy
    got = need(n, H, C, K, temp, bf, True)
    words = max(256 * MB // (rows * e), 2048)
    piece = rows * min(up(words, 256), up(C, 256)) * e
    whole = C <= words
    most = least + copy + max(64 * MB, rows * H * 4) + 128 * MB + piece + piece // e // 16
    if bf:
        most += 2 * piece if whole else piece
    assert got <= most
    # of one piece at least half is taken: the pieces are of equal width
    assert got >= least - 2 * SLACK + copy + rows * H * 4 + (piece if whole else piece // 2)


def test_a_million_rows_take_more_than_pieces_of_256_mb():
    """What a caller has to have at the largest n: 2048 words of dL/dz and of z."""
    _ensure_built()
    n, C = 1 << 20, 2048
    assert need(n, 1024, C, 0, 1.0, True, True) >= n * C * (2 + 4) + n * 1024 * (2 + 4)
    assert need(n, 64, C, 0, 1.0, False, True) >= n * C * 4
