"""MXFP4 rows: quantisation and back against the format's definition in 64 bits, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2606_19025_amd import binding as B
from paper_2606_19025_amd.layer import mxfp4_dequantize, mxfp4_quantize

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def stride(cols):
    return -(-cols // 128) * 4


def oracle(x):
    """(codes, scales, values) of 64-bit rows by the definition: distances to the grid."""
    rows, cols = x.shape
    b = x.reshape(rows, -1, 32)
    top = np.abs(b).max(axis=2)
    bad = ~np.isfinite(b).all(axis=2)
    e = np.frexp(np.where(bad, 1.0, top))[1] - 1
    s = np.where(top == 0, 0, np.maximum(0, e - 2 + 127))
    v = np.where(bad[..., None], 0.0, b) * np.exp2(127.0 - s)[..., None]
    dist = np.abs(np.abs(v)[..., None] - GRID)
    dist[..., 1::2] += 1e-9  # ties to the even code: distances are multiples of 2^-26 here or exact
    code = dist.argmin(axis=-1)
    values = np.copysign(GRID[code], v) * np.exp2(s - 127.0)[..., None]
    code = code + 8 * np.signbit(v)
    code[bad], s[bad], values[bad] = 0, 255, np.nan
    code = code.reshape(rows, cols).astype(np.uint8)
    scales = np.zeros((rows, stride(cols)), np.uint8)
    scales[:, : cols // 32] = s
    return code[:, 0::2] | code[:, 1::2] << 4, scales, values.reshape(rows, cols)


def run(x, n_rows=None):
    """The pair and the values, on buffers with a canary row behind the last."""
    rows, cols = x.shape
    codes = torch.full((rows + 1, cols // 2), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows + 1, stride(cols)), 0xA5, dtype=torch.uint8, device="cuda")
    back = torch.full((rows + 1, cols), 7.0, dtype=x.dtype, device="cuda")
    mxfp4_quantize(x, out=(codes[:rows], scales[:rows]), n_rows=n_rows)
    mxfp4_dequantize(codes[:rows], scales[:rows], x.dtype, out=back[:rows], n_rows=n_rows)
    torch.cuda.synchronize()
    return codes.cpu().numpy(), scales.cpu().numpy(), back.double().cpu().numpy()


def compare(x):
    codes, scales, back = run(x)
    rc, rs, rv = oracle(x.double().cpu().numpy())
    assert np.array_equal(scales[:-1], rs)
    assert np.array_equal(codes[:-1], rc)
    assert np.array_equal(back[:-1], rv, equal_nan=True)
    assert (codes[-1] == 0xA5).all() and (scales[-1] == 0xA5).all() and (back[-1] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 64), (257, 96), (5, 704), (33, 1024), (1000, 160)])
def test_quantize_is_the_definition(gpu_lib, rows, cols, dtype):
    g = torch.Generator().manual_seed(rows + cols)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(6 * torch.randn(rows, 1, generator=g))
    compare(x.to(DT[dtype]).cuda())


@pytest.mark.gpu
def test_every_bf16_value(gpu_lib):
    """Each finite bf16 bit pattern, once as its block's largest magnitude and once under each
    of eight larger ones (ties, underflow to zero, subnormals, the largest finite value)."""
    bits = np.arange(65536, dtype=np.uint32) << 16
    v = bits.view(np.float32)
    v = v[np.isfinite(v)]
    blocks = []
    for up in (0, 1, 2, 3, 4, 8, 60, 126):
        top = np.minimum(np.abs(v.astype(np.float64)) * 2.0 ** up, 3.3e38)
        b = np.zeros((v.size, 32))
        b[:, 3], b[:, 20] = v, np.where(np.abs(v) < top, top, 0.0)
        blocks.append(b)
    x = torch.from_numpy(np.concatenate(blocks)).to(torch.bfloat16)
    compare(x.cuda())
    compare(x.float().cuda())


@pytest.mark.gpu
def test_borders_of_the_grid(gpu_lib):
    """fp32 values on each border between two codes and one step to either side of it."""
    mid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0], np.float32)
    v = np.concatenate([mid, np.nextafter(mid, np.float32(0)), np.nextafter(mid, np.float32(9))])
    for e in (-120, -64, -63, 0, 90):
        b = np.zeros((2, 32), np.float32)
        b[0, : v.size], b[1, : v.size] = v, -v
        b[:, 31] = 7.5
        compare(torch.from_numpy(np.ldexp(b, e)).cuda())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_blocks_that_are_not_finite(gpu_lib, dtype):
    """An infinity or a NaN makes its own block NaN, and no other."""
    x = torch.randn(4, 256)
    x[0, 40], x[1, 200], x[2, 0], x[2, 255] = float("inf"), float("nan"), float("-inf"), 3.0
    x[3] = 0.0
    compare(x.to(DT[dtype]).cuda())


@pytest.mark.gpu
@pytest.mark.parametrize("n", [-3, 0, 1, 17, 40, 99])
def test_rows_past_the_device_count(gpu_lib, n):
    """Only the first *n_rows rows are read and written."""
    x = torch.randn(40, 96, device="cuda")
    x[max(0, min(n, 40)):] = float("nan")
    codes, scales, back = run(x, torch.tensor([n], dtype=torch.int32, device="cuda"))
    m = max(0, min(n, 40))
    rc, rs, rv = oracle(x[:m].double().cpu().numpy()) if m else (codes[:0], scales[:0], back[:0])
    assert np.array_equal(codes[:m], rc) and np.array_equal(scales[:m], rs) and np.array_equal(back[:m], rv)
    assert (codes[m:] == 0xA5).all() and (scales[m:] == 0xA5).all() and (back[m:] == 7).all()


@pytest.mark.gpu
def test_count_of_rows_is_one_value(gpu_lib):
    x = torch.randn(4, 64, device="cuda")
    one = torch.tensor(2, dtype=torch.int32, device="cuda")
    pair = mxfp4_quantize(x, n_rows=one)
    mxfp4_dequantize(*pair, n_rows=one)
    for bad in (torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"),
                torch.zeros(1, dtype=torch.int32), 3):
        with pytest.raises(ValueError):
            mxfp4_quantize(x, n_rows=bad)
        with pytest.raises(ValueError):
            mxfp4_dequantize(*pair, n_rows=bad)


@pytest.mark.gpu
def test_round_trip_keeps_its_values_and_replays(gpu_lib):
    """Values of the format come back as they are; a captured pass follows its input."""
    x = torch.randn(64, 256, device="cuda")
    q = mxfp4_quantize(x)
    v = mxfp4_dequantize(*q, torch.float32)
    again = mxfp4_quantize(v)
    assert torch.equal(mxfp4_dequantize(*again, torch.float32), v)
    live, out = x.clone(), torch.empty_like(x)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p = mxfp4_quantize(live)
        mxfp4_dequantize(*p, torch.float32, out=out)
    for seed in (1, 2, 3):
        live.copy_(torch.randn(64, 256, generator=torch.Generator().manual_seed(seed)))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, mxfp4_dequantize(*mxfp4_quantize(live), torch.float32))


@pytest.mark.gpu
def test_new_buffers_are_of_the_calls_stream(gpu_lib):
    """Buffers that a call makes on another stream than the current one are not memory that the
    current stream has yet to write: the latter is kept busy, then fills tensors of the same sizes,
    which are dropped at once (their memory is the next to be given out on that stream)."""
    from paper_2606_19025_amd.layer import InferenceMoELayer, LayerNorm, ResidentMoELayer
    T, d, k, H = 64, 512, 2, 256
    g = torch.Generator(device="cuda").manual_seed(5)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda").mul(0.3).bfloat16()
    x, dy, w = n(T, d), n(T, d), torch.ones(d, device="cuda")
    router, gu, dn = n(8, d), n(8, 2 * H, d), n(8, d, H)
    big, res = n(2048, 2048), torch.ones(8, dtype=torch.uint8)
    pair = mxfp4_quantize(big)
    norms, few = [LayerNorm(T, d, bias=False) for _ in range(3)], lambda: InferenceMoELayer(k, res, router, gu, dn)
    layers, fews = [ResidentMoELayer(T, d, 8, k, H, res) for _ in range(3)], [few() for _ in range(3)]
    for N in norms:
        N.forward(x, w)

    def step(R, stream):
        y = R.forward(x, router, gu, dn, stream=stream)
        return [y, R.backward(dy, x, router, gu, dn, stream=stream), R.dw_gate_up]

    calls = [lambda i, s: list(mxfp4_quantize(big, stream=s)),
             lambda i, s: [mxfp4_dequantize(*pair, stream=s)],
             lambda i, s: [norms[i].backward(dy, x, w, stream=s), norms[i].dw],
             lambda i, s: [fews[i].few(x, stream=s), fews[i].logits], lambda i, s: step(layers[i], s)]
    side, busy = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    for call in calls:
        want = [v.clone() for v in call(0, None)]
        for i, s in ((1, side), (2, side.cuda_stream)):
            torch.cuda.synchronize()
            for _ in range(8):
                busy @ busy
            sizes = [1 << b for b in range(9, 24)] + [3 << b for b in range(9, 22)]
            junk = [torch.full((m,), 0x5A, dtype=torch.uint8, device="cuda") for m in sizes]
            del junk
            got = call(i, s)
            torch.cuda.synchronize()
            assert all(torch.equal(u, v) for u, v in zip(got, want))


def test_mx_refusals():
    if torch.cuda.device_count() > 0:
        pytest.skip("host-only rejection test: runs where no GPU is visible")
    L, p = B.lib(), 256  # a fake, never dereferenced address
    assert [B.moe_mxfp4_scale_stride(c) for c in (-1, 0, 32, 128, 160, 704)] == [0, 0, 4, 4, 8, 24]
    q = lambda x=p, dt=B.MOE_F32, rows=2, cols=64, c=p, s=p: L.moe_mxfp4_quantize(x, dt, rows, cols, None, c, s, None)
    d = lambda x=p, dt=B.MOE_F32, rows=2, cols=64, c=p, s=p: L.moe_mxfp4_dequantize(c, s, dt, rows, cols, None, x, None)
    for f in (q, d):
        assert f(dt=5) == -2 and f(cols=48) == -2 and f(x=p + 4) == -2 and f(c=p + 8) == -2
        assert f(rows=-1) == -1 and f(cols=0) == -1 and f(x=None) == -1 and f(c=None) == -1 and f(s=None) == -1
        assert f(rows=2 ** 31 - 1, cols=2 ** 31 - 32) == -2
    for bad in (torch.zeros(4, 64), torch.zeros(32), None):
        with pytest.raises(ValueError):
            mxfp4_quantize(bad)


def test_mx_more_words_than_a_grid():
    """A grid holds fewer than 2^32 threads of four words each: past that the call is refused (with
    an unaligned x, whose check comes later and ends the calls that may go on here)."""
    if torch.cuda.device_count() > 0:
        pytest.skip("host-only rejection test: runs where no GPU is visible")
    L, p = B.lib(), 256  # a fake, never dereferenced address
    for rows, cols, many in ((2 ** 22 - 1, 2 ** 15, False), (2 ** 24 - 1, 2 ** 13, False), (2 ** 22, 2 ** 15, True),
                             (2 ** 24, 2 ** 13, True), (2 ** 31 - 1, 32, False), (2 ** 31 - 1, 64, True)):
        for r in (L.moe_mxfp4_quantize(p + 4, B.MOE_BF16, rows, cols, None, p, p, None),
                  L.moe_mxfp4_dequantize(p, p, B.MOE_BF16, rows, cols, None, p + 4, None)):
            assert r == -2 and ("too many" in B.moe_last_error()) == many, (rows, cols, B.moe_last_error())


def test_the_oracle_of_these_tests():
    """By hand: 5 is a tie (4 and 6: the even code, 4), 7.9 saturates, the scale is 2^(2 - 2)."""
    x = np.zeros((1, 32))
    x[0, :6] = [5, -7.9, 0.25, 0.75, -2.5, 1.3]
    c, s, v = oracle(x)
    assert s[0, 0] == 127 and list(v[0, :6]) == [4, -6, 0, 1, -2, 1.5]
    assert list(c[0, :3]) == [0xF6, 0x20, 0x3C]
