"""What the linear head's forward asks for beside its inputs."""
import ctypes as C

import pytest

from paper_2606_19025_amd import binding as B


def size(N, d, V, dtype):
    L, p = B.lib(), 1 << 12  # (an address that is never read)
    return L.moe_xent_fwd_workspace_size(C.byref(B.moe_xent(
        dtype=dtype, N=N, d=d, V=V, scale=1.0, x=p, w=p, labels=p, loss=p, lse=p, total=p)))


@pytest.mark.parametrize("dtype,N,d,V,columns", [
    # enough tiles of 256 x 256 (bf16) or 64 x 128 (fp32) for every CU several times over
    (B.MOE_BF16, 8192, 2048, 49152, 128), (B.MOE_BF16, 65536, 1024, 131072, 128),
    (B.MOE_F32, 8192, 2048, 49152, 64), (B.MOE_F32, 4000, 512, 32003, 64),
    # few: the smallest tiles at most
    (B.MOE_BF16, 5, 64, 700, 32), (B.MOE_F32, 33, 64, 257, 32), (B.MOE_BF16, 24, 2048, 49152, 32)])
def test_forward_asks_for_the_partials_of_its_tiles(dtype, N, d, V, columns):
    """Two words of a half tile's columns for each token, beside the copy of the tokens' rows, a few
    numbers for each and less than 16 roundings to 256 bytes."""
    partials = 8 * N * 2 * -(-V // (2 * columns))
    rows = N * d * (2 if dtype == B.MOE_BF16 else 4)
    got = size(N, d, V, dtype)
    assert rows < got <= rows + partials + 32 * N + 16 * 256
