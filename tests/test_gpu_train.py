"""The training step's kernels on the GPU against the 64-bit oracle: the 8-bit
block format bit for bit, products within the error of fp32 sums, the norm,
and the AdamW step with fp32 and 8-bit states; odd sizes, strides and
alignments, entries that are not finite, streams and graph replays."""

import math

import numpy as np
import pytest

from gpu_util import torch_dev
from oracle import train as O
from paper_2609_23898_amd import cerar as C
from paper_2609_23898_amd import train as T

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24


def dtype_of(name):
    torch, _ = torch_dev()
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def device(a, name="f32", shift=0, pad=0):
    """A matrix or vector on the device as `name`, `shift` entries into its
    buffer and with rows `pad` entries apart; and the values it holds there (float64)."""
    torch, dev = torch_dev()
    a = np.asarray(a, dtype=np.float32)
    rows, cols = a.shape if a.ndim == 2 else (1, a.shape[0])
    buf = torch.full((rows * (cols + pad) + shift + 8,), 7.0, dtype=dtype_of(name), device=dev)
    t = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.from_numpy(a.reshape(rows, cols)).to(dev))
    if a.ndim == 1:
        t = t.view(-1)
    return t, t.double().cpu().numpy()


def host8(t):
    torch, _ = torch_dev()
    return t.view(torch.uint8).cpu().numpy()


def values(b):
    return O.matrix(host8(b.codes), host8(b.scales), b.fmt)


def guarded_blocks(rows, cols, fmt):
    """A Blocks inside larger buffers of 0xA5, and a check that nothing beside it was written."""
    torch, dev = torch_dev()
    ld = O.up(cols, 128)
    groups = -(-ld // 512)
    code_buf = torch.full((rows * ld + 256,), 0xA5, dtype=torch.uint8, device=dev)
    scale_buf = torch.full((groups * rows * 4 + 64,), 0xA5, dtype=torch.uint8, device=dev)
    f8 = torch.float8_e4m3fn if fmt == "e4m3" else torch.float8_e5m2
    b = T.Blocks(code_buf[128:128 + rows * ld].view(rows, ld).view(f8),
                 scale_buf[32:32 + groups * rows * 4].view(groups, rows, 4), cols)

    def check():
        for buf, lo, n in ((code_buf, 128, rows * ld), (scale_buf, 32, groups * rows * 4)):
            assert bool((buf[:lo] == 0xA5).all()) and bool((buf[lo + n:] == 0xA5).all())

    return b, check


def wild(rng, rows, cols):
    """Rows of very different sizes, blocks of zeros, exact ties of the largest value."""
    x = rng.standard_normal((rows, cols)) * 2.0 ** rng.uniform(-30, 20, (rows, 1))
    x[rng.random((rows, cols)) < 0.05] = 0.0
    if rows > 3:
        x[1] = 0.0
        x[2, 0] = 448.0
        x[3] = 1.75 * 2.0 ** rng.integers(-8, 8)
    return x


# --- quantize ----------------------------------------------------------------------

@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (1, 700), (7, 130), (127, 129), (128, 128), (129, 127),
                                       (260, 515), (5, 1025), (1000, 3)])
@pytest.mark.parametrize("fmt,tile", [("e4m3", False), ("e5m2", False), ("e4m3", True), ("e5m2", True)])
@pytest.mark.parametrize("name,shift,pad", [("f32", 0, 0), ("bf16", 0, 0), ("f32", 1, 3), ("bf16", 1, 5)])
def test_quantize_matches_oracle(rows, cols, fmt, tile, name, shift, pad):
    rng = np.random.default_rng(rows * 1000 + cols)
    x, xv = device(wild(rng, rows, cols), name, shift, pad)
    r, check_r = guarded_blocks(rows, cols, fmt)
    c, check_c = guarded_blocks(cols, rows, fmt)
    T.quantize_blocks(x, rows=r, cols=c, tile=tile)
    (rc, rk), (cc, ck) = O.quantize(xv, fmt, tile)
    for b, codes, k, check in ((r, rc, rk, check_r), (c, cc, ck, check_c)):
        np.testing.assert_array_equal(host8(b.scales), O.lay_scales(k))
        np.testing.assert_array_equal(host8(b.codes), codes)
        check()
    for only in ("rows", "cols"):                       # either form alone
        b, check = guarded_blocks(*((rows, cols) if only == "rows" else (cols, rows)), fmt)
        T.quantize_blocks(x, **{only: b}, tile=tile)
        both = r if only == "rows" else c
        np.testing.assert_array_equal(host8(b.codes), host8(both.codes))
        np.testing.assert_array_equal(host8(b.scales), host8(both.scales))
        check()


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("tile", [False, True])
def test_quantize_extremes(fmt, tile):
    """NaN, infinities, the largest and smallest fp32 values, subnormal ones and
    signed zeros; a block's scale comes from its finite entries."""
    rng = np.random.default_rng(5)
    x = rng.standard_normal((130, 260))
    x[0, :8] = [np.nan, np.inf, -np.inf, -0.0, 1.0, 0.0, 3e38, -3.4028235e38]
    x[1] = np.nan
    x[2, 128:256] = np.inf
    x[3, :128] = 2.0 ** -149
    x[4, :128] = 2.0 ** rng.uniform(-149, -120, 128)
    x[5, 0:128:3] = -2.0 ** -140
    t, xv = device(x)
    r, _ = guarded_blocks(130, 260, fmt)
    c, _ = guarded_blocks(260, 130, fmt)
    T.quantize_blocks(t, rows=r, cols=c, tile=tile)
    for b, (codes, k) in zip((r, c), O.quantize(xv, fmt, tile)):
        np.testing.assert_array_equal(host8(b.scales), O.lay_scales(k))
        got = host8(b.codes)
        nan = np.isnan(O.code_values(fmt)[codes])
        np.testing.assert_array_equal(np.isnan(O.code_values(fmt)[got]), nan)
        np.testing.assert_array_equal(got[~nan], codes[~nan])


def test_quantize_nothing():
    torch, dev = torch_dev()
    for rows, cols in ((0, 5), (5, 0)):
        T.quantize_blocks(torch.zeros((rows, cols), device=dev), rows=T.Blocks.empty(rows, cols))


# --- products -----------------------------------------------------------------------

def random_blocks(rng, rows, cols, fmt, lo=110, hi=144):
    """Codes of every finite value and scales over 2^-17 .. 2^16."""
    torch, dev = torch_dev()
    ld = O.up(cols, 128)
    top = 0x7F if fmt == "e4m3" else 0x7C
    codes = rng.integers(0, top, (rows, ld)) | rng.integers(0, 2, (rows, ld)) << 7
    codes[:, cols:] = 0
    scales = O.lay_scales(rng.integers(lo, hi, (rows, ld // 128)) - 127)
    f8 = torch.float8_e4m3fn if fmt == "e4m3" else torch.float8_e5m2
    return T.Blocks(torch.from_numpy(codes.astype(np.uint8)).to(dev).view(f8), torch.from_numpy(scales).to(dev), cols)


def out_buffer(M, N, name, pad=0, shift=0, fill=None):
    """(tensor, its whole buffer): rows pad entries apart, the buffer filled with 7."""
    torch, dev = torch_dev()
    buf = torch.full((M * (N + pad) + shift + 64,), 7.0, dtype=dtype_of(name), device=dev)
    t = buf[shift:shift + M * (N + pad)].view(M, N + pad)[:, :N]
    if fill is not None:
        t.copy_(torch.from_numpy(np.asarray(fill)).to(dev))
    return t, buf


def workspace(M, N, K, linear=False):
    torch, dev = torch_dev()
    return torch.empty(T.matmul_workspace_bytes(M, N, K, linear), dtype=torch.uint8, device=dev)


def sum_bound(A, B):
    """The error of sums of K products in fp32 in any order, each addition off by
    at most one unit in the last place (2^-23): K 2^-23 sum |a b|."""
    return A.shape[1] * 2.0 ** -23 * (np.abs(A) @ np.abs(B).T)


def check_product(got, A, B, name, start=0.0):
    ref = A @ B.T + start
    tol = sum_bound(A, B) + 2 * U32 * (np.abs(ref) + np.abs(start))
    if name == "bf16":
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)
    err = np.abs(got - ref)
    assert np.isfinite(got).all() and (err <= tol).all(), (err / np.maximum(tol, 1e-300)).max()


SHAPES = [(1, 1, 1), (1, 257, 130), (2, 64, 128), (7, 1000, 2050), (15, 33, 515), (16, 16, 129), (17, 130, 1024), (31, 65, 640),
          (33, 31, 1500), (45, 513, 257), (64, 64, 128), (65, 129, 384), (100, 300, 700), (128, 128, 512), (129, 255, 896),
          (257, 260, 127), (300, 1, 300), (256, 512, 1280), (511, 383, 2049), (1030, 270, 200)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("name,add", [("bf16", False), ("f32", False), ("f32", True)])
def test_matmul_matches_oracle(M, N, K, fa, fb, name, add):
    rng = np.random.default_rng(M * 7 + N * 3 + K)
    a, b = random_blocks(rng, M, K, fa), random_blocks(rng, N, K, fb)
    A, B = values(a), values(b)
    start = (rng.standard_normal((M, N)) * np.abs(A @ B.T).mean()).astype(np.float32) if add else None
    pad, shift = [(0, 0), (5, 1), (8, 0)][(M + N) % 3]
    out, buf = out_buffer(M, N, name, pad, shift, start)
    T.matmul_blocks(a, b, out, workspace(M, N, K), accumulate=add)
    check_product(out.double().cpu().numpy(), A, B, name, 0.0 if start is None else start.astype(np.float64))
    whole = buf.double().cpu().numpy()
    beside = np.ones(whole.shape, dtype=bool)
    for m in range(M):
        beside[shift + m * (N + pad):shift + m * (N + pad) + N] = False
    assert (whole[beside] == 7.0).all()


def group_bound(A, B):
    """The 8-bit instructions' sums: each product loses less than 2^-12 of the
    largest of its group of eight neighbours (13 bits below that one's leading
    bit are kept, and a product's leading bit is its first or second), and the
    groups' sums are added in fp32."""
    K = A.shape[1]
    worst = np.zeros((A.shape[0], B.shape[0]))
    for g in range(0, K, 8):
        worst += (np.abs(A)[:, None, g:g + 8] * np.abs(B)[None, :, g:g + 8]).max(2)
    return 8 * 2.0 ** -12 * worst + sum_bound(A, B)


SUMS = [(1, 500, 4096), (40, 300, 2048), (64, 130, 2048), (70, 200, 1024), (129, 257, 640), (130, 120, 16384), (4352, 4480, 256),
        (4200, 4300, 384), (203, 12108, 10240), (3000, 3000, 16384)]


@pytest.mark.parametrize("M,N,K", SUMS)
@pytest.mark.parametrize("name,add", [("f32", False), ("f32", True), ("bf16", False)])
def test_fp32_sums_keep_a_term_far_below_its_neighbours(M, N, K, name, add):
    """Eight neighbouring terms are 1, -1, 2^-16 and zeros.  Groups of them add up to K 2^-19 without a
    rounding in fp32 (multiples of 2^-16 below 2^8); the 8-bit instruction loses the small terms.  K is a
    power of two times 5 at most, so that bf16 holds the result.  Tiles of either size, whole K and K in
    parts, whole tiles and their edges, and few rows."""
    torch, dev = torch_dev()
    codes = torch.zeros((1, K), dtype=torch.uint8, device=dev)
    codes[:, 0::8], codes[:, 3::8], codes[:, 6::8] = 0x38, 0x38, 0x02        # 1, 1, 2^-8
    signed = codes.clone()
    signed[:, 3::8] = 0xB8                                                   # -1

    def operand(codes, rows, seed):
        gen = torch.Generator(device=dev).manual_seed(seed)
        k = torch.randint(-3, 4, (rows,), device=dev, generator=gen)
        scales = torch.zeros((-(-K // 512), rows, 4), dtype=torch.uint8, device=dev)
        for b in range(K // 128):
            scales[b // 4, :, b % 4] = (k + 127).to(torch.uint8)
        return T.Blocks(codes.expand(rows, K).contiguous().view(torch.float8_e4m3fn), scales, K), 2.0 ** k.double()

    (a, fa), (b, fb) = operand(codes, M, 1), operand(signed, N, 2)
    want = fa[:, None] * fb[None, :] * (K / 2.0 ** 19)
    out, _ = out_buffer(M, N, name)
    out.zero_()
    T.matmul_blocks(a, b, out, workspace(M, N, K), accumulate=add)
    assert torch.equal(out.double(), want)
    if M > 64 and not add and name == "f32":
        T.matmul_blocks(a, b, out, workspace(M, N, K), fast_sums=True)
        assert not bool((out.double() == want).any())


@pytest.mark.parametrize("M,N,K", [(30, 70, 8192), (100, 90, 1000), (130, 120, 16000), (700, 530, 9000), (1030, 270, 2049),
                                   (3000, 3000, 16384)])
def test_fp32_sums_of_long_rows_are_those_of_fp32(M, N, K):
    """Each of K additions rounds by 2^-24 of a partial sum at most, which is no larger than the
    result in the mean over results: 2^-24 sqrt(K) of it in all, if the roundings are
    independent, where the 8-bit instruction is off by 1.5e-5 to 5e-5 whatever K."""
    torch, dev = torch_dev()
    rng = np.random.default_rng(K)
    a, b = random_blocks(rng, M, K, "e5m2", 126, 129), random_blocks(rng, N, K, "e4m3", 126, 129)
    out, _ = out_buffer(M, N, "f32")
    T.matmul_blocks(a, b, out, workspace(M, N, K))
    rows = np.unique(rng.integers(0, M, 150))
    ref = values(a)[rows] @ values(b).T
    err = out.double().cpu().numpy()[rows] - ref
    assert math.sqrt((err ** 2).mean()) <= U32 * math.sqrt(K) * math.sqrt((ref ** 2).mean())


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
def test_fast_sums_match_oracle(M, N, K, fa, fb):
    rng = np.random.default_rng(M * 5 + N + K)
    a, b = random_blocks(rng, M, K, fa), random_blocks(rng, N, K, fb)
    A, B = values(a), values(b)
    ref, tol = A @ B.T, group_bound(A, B)
    for name, start in (("f32", None), ("bf16", None), ("f32", rng.standard_normal((M, N)).astype(np.float32))):
        out, _ = out_buffer(M, N, name, pad=1, fill=start)
        T.matmul_blocks(a, b, out, workspace(M, N, K), accumulate=start is not None, fast_sums=True)
        got = out.double().cpu().numpy()
        want = ref if start is None else ref + start
        slack = (2.0 ** -8 * (np.abs(want) + tol) if name == "bf16" else 2 * U32 * np.abs(want))
        assert (np.abs(got - want) <= tol + slack).all(), (np.abs(got - want) / (tol + slack)).max()
    x, xv = device(wild(rng, M, K), "bf16", shift=1, pad=2)
    (codes, k), _ = O.quantize(xv, "e4m3")
    X = O.matrix(codes, O.lay_scales(k), "e4m3")
    out, _ = out_buffer(M, N, "bf16")
    T.linear_blocks(x, b, out, workspace(M, N, K, True), fast_sums=True)
    want, tol = X @ B.T, group_bound(X, B)
    assert (np.abs(out.double().cpu().numpy() - want) <= tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)).all()


@pytest.mark.parametrize("M,N,K,fast", [(4200, 4300, 130, True), (4200, 4300, 300, True), (4111, 4353, 513, True),
                                        (4200, 4300, 300, False), (5000, 270, 1030, True), (700, 530, 9000, True),
                                        (700, 530, 9000, False), (130, 120, 16000, True), (130, 120, 16000, False)])
@pytest.mark.parametrize("name,add", [("bf16", False), ("f32", False), ("f32", True)])
def test_large_matmul_matches_oracle(M, N, K, fast, name, add):
    """More tiles than compute units, and few tiles over a long K: whole rows and columns of the result."""
    torch, dev = torch_dev()
    rng = np.random.default_rng(M + N + K)
    a, b = random_blocks(rng, M, K, "e4m3"), random_blocks(rng, N, K, "e5m2" if add else "e4m3")
    start = rng.standard_normal((M, N)).astype(np.float32) * 1e4 if add else None
    out, buf = out_buffer(M, N, name, pad=3, shift=1, fill=start)
    T.matmul_blocks(a, b, out, workspace(M, N, K), accumulate=add, fast_sums=fast)
    A, B, got = values(a), values(b), out.double().cpu().numpy()
    for rows, cols in ((np.unique(rng.integers(0, M, 60)), np.arange(N)), (np.arange(M), np.unique(rng.integers(0, N, 60)))):
        ref = A[rows] @ B[cols].T + (start[np.ix_(rows, cols)].astype(np.float64) if add else 0.0)
        tol = (group_bound if fast else sum_bound)(A[rows], B[cols]) + 4 * U32 * np.abs(ref)
        if add:
            tol = tol + 2 * U32 * np.abs(start[np.ix_(rows, cols)])
        if name == "bf16":
            tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)
        assert (np.abs(got[np.ix_(rows, cols)] - ref) <= tol).all()
    whole = buf[1:1 + M * (N + 3)].view(M, N + 3)
    assert bool((buf[:1] == 7).all()) and bool((whole[:, N:] == 7).all()) and bool((buf[1 + M * (N + 3):] == 7).all())


def bound_of_few(A, B, fast):
    """group_bound or sum_bound where A or B has few rows, one of them at a time."""
    if B.shape[0] < A.shape[0]:
        return bound_of_few(B, A, fast).T
    B = np.abs(B)
    tol = np.zeros((A.shape[0], B.shape[0]))
    for i, a in enumerate(np.abs(A)):
        tol[i] = A.shape[1] * 2.0 ** -23 * (B @ a)
        if fast:
            tol[i] += 8 * 2.0 ** -12 * np.maximum.reduceat(B * a, np.arange(0, len(a), 8), axis=1).sum(1)
    return tol


@pytest.mark.parametrize("M,N,K,pad,fast", [
    (4352, 4480, 300, 0, True), (4352, 4480, 300, 0, False),         # 256 x 256: rows on cache lines, whole and edge columns
    (4400, 4300, 130, 52, True), (4400, 4300, 130, 52, False),       # and with a padded row, edges both ways
    (4400, 4300, 100, 0, True), (4400, 4352, 128, 0, True),          # one block of K
    (5345, 1075, 12235, 1, True), (203, 12108, 9999, 4, False), (203, 12108, 9999, 0, True),   # 256 x 256 with K in parts
    (640, 768, 700, 0, True), (640, 768, 700, 0, False), (700, 650, 515, 118, True)])          # 128 x 128 on cache lines
@pytest.mark.parametrize("name,add", [("bf16", False), ("f32", False), ("f32", True)])
def test_every_way_that_tiles_leave_matches_oracle(M, N, K, pad, fast, name, add):
    """Whole tiles and edges, stored past the L2 and through it, from either size of tile, and joined."""
    rng = np.random.default_rng(M + N + K)
    a, b = random_blocks(rng, M, K, "e5m2" if add else "e4m3"), random_blocks(rng, N, K, "e4m3")
    start = rng.standard_normal((M, N)).astype(np.float32) * 1e4 if add else None
    out, buf = out_buffer(M, N, name, pad=pad, fill=start)
    T.matmul_blocks(a, b, out, workspace(M, N, K), accumulate=add, fast_sums=fast)
    A, B, got = values(a), values(b), out.double().cpu().numpy()
    count = 40 if K < 1000 else 3
    for rows, cols in ((np.unique(rng.integers(0, M, count)), np.arange(N)), (np.arange(M), np.unique(rng.integers(0, N, count)))):
        ref = A[rows] @ B[cols].T + (start[np.ix_(rows, cols)].astype(np.float64) if add else 0.0)
        tol = bound_of_few(A[rows], B[cols], fast) + 4 * U32 * np.abs(ref)
        if add:
            tol = tol + 2 * U32 * np.abs(start[np.ix_(rows, cols)])
        if name == "bf16":
            tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)
        assert (np.abs(got[np.ix_(rows, cols)] - ref) <= tol).all()
    assert bool((buf[:M * (N + pad)].view(M, N + pad)[:, N:] == 7).all()) and bool((buf[M * (N + pad):] == 7).all())


@pytest.mark.parametrize("M,N", [(100, 70), (300, 300), (4400, 4352)])
@pytest.mark.parametrize("fast", [False, True])
def test_more_rows_of_no_columns(M, N, fast):
    torch, dev = torch_dev()
    a, b = T.Blocks.empty(M, 0), T.Blocks.empty(N, 0)
    for name in ("f32", "bf16"):
        out, _ = out_buffer(M, N, name, pad=1)
        if name == "f32":
            T.matmul_blocks(a, b, out, workspace(M, N, 0), accumulate=True, fast_sums=fast)
            assert bool((out == 7).all())
        T.matmul_blocks(a, b, out, workspace(M, N, 0), fast_sums=fast)
        assert bool((out == 0).all())
        out.fill_(7)
        T.linear_blocks(torch.empty((M, 0), device=dev), b, out, workspace(M, N, 0, True), fast_sums=fast)
        assert bool((out == 0).all())


@pytest.mark.parametrize("lo,hi", [(1, 3), (240, 248)])
@pytest.mark.parametrize("M,N,K", [(30, 90, 400), (70, 90, 400), (300, 270, 700)])
def test_fast_sums_of_scales_at_both_ends(M, N, K, lo, hi):
    rng = np.random.default_rng(4)
    a, b = random_blocks(rng, M, K, "e4m3", lo, hi), random_blocks(rng, N, K, "e4m3", 254 - hi, 254 - lo)
    out, _ = out_buffer(M, N, "f32")
    T.matmul_blocks(a, b, out, workspace(M, N, K), fast_sums=True)
    A, B = values(a), values(b)
    ref = A @ B.T
    assert (np.abs(out.double().cpu().numpy() - ref) <= group_bound(A, B) + 2 * U32 * np.abs(ref)).all()


@pytest.mark.parametrize("M,N,K", [(4352, 4480, 300), (203, 12108, 9999), (8192, 4096, 2048)])
def test_large_products_repeat_their_bits(M, N, K):
    """Also after calls on other operands, whose codes the chip's caches then hold."""
    torch, dev = torch_dev()
    rng = np.random.default_rng(8)
    a, b = random_blocks(rng, M, K, "e4m3"), random_blocks(rng, N, K, "e4m3")
    other = random_blocks(rng, M, K, "e4m3")
    ws, out, scratch = workspace(M, N, K), out_buffer(M, N, "bf16")[0], out_buffer(M, N, "bf16")[0]
    first = {}
    for k in range(8):
        fast = k % 2 == 1
        T.matmul_blocks(other, b, scratch, ws, fast_sums=fast)
        out.fill_(7)
        T.matmul_blocks(a, b, out, ws, fast_sums=fast)
        assert torch.equal(first.setdefault(fast, out.clone()), out)


def test_matmul_applies_each_scale_to_its_block():
    """One code of one in each operand's row and column: entry (m, n) is the sum
    over blocks of 2^(ka + kb), exact in fp32, whatever the scales' layout."""
    torch, dev = torch_dev()
    rng = np.random.default_rng(3)
    for M, N, kb in ((40, 50, 6), (300, 270, 9), (1, 70, 13)):
        K = kb * 128
        ops = []
        for rows in (M, N):
            codes = np.zeros((rows, K), dtype=np.uint8)
            codes[:, ::128] = 0x38                       # 1.0 in e4m3
            k = rng.integers(-5, 6, (rows, kb))
            ops.append((T.Blocks(torch.from_numpy(codes).to(dev).view(torch.float8_e4m3fn),
                                 torch.from_numpy(O.lay_scales(k)).to(dev), K), 2.0 ** k.astype(float)))
        for fast in (False, True):
            out, _ = out_buffer(M, N, "f32")
            T.matmul_blocks(ops[0][0], ops[1][0], out, workspace(M, N, K), fast_sums=fast)
            np.testing.assert_array_equal(out.double().cpu().numpy(), ops[0][1] @ ops[1][1].T)


def test_matmul_of_nothing():
    torch, dev = torch_dev()
    out, buf = out_buffer(3, 4, "f32")
    T.matmul_blocks(T.Blocks.empty(3, 0), T.Blocks.empty(4, 0), out, workspace(3, 4, 0))
    assert bool((out == 0).all())
    out, _ = out_buffer(3, 4, "f32")
    T.matmul_blocks(T.Blocks.empty(3, 0), T.Blocks.empty(4, 0), out, workspace(3, 4, 0), accumulate=True)
    assert bool((out == 7).all())
    T.linear_blocks(torch.empty((3, 0), device=dev), T.Blocks.empty(4, 0), out, workspace(3, 4, 0, True))
    assert bool((out == 0).all())
    T.matmul_blocks(T.Blocks.empty(0, 50), T.Blocks.empty(4, 50), torch.empty((0, 4), device=dev), workspace(0, 4, 50))
    T.matmul_blocks(T.Blocks.empty(3, 50), T.Blocks.empty(0, 50), torch.empty((3, 0), device=dev), workspace(3, 0, 50))
    T.linear_blocks(torch.empty((0, 50), device=dev), T.Blocks.empty(4, 50), torch.empty((0, 4), device=dev),
                    workspace(0, 4, 50, True))
    torch.cuda.synchronize()


@pytest.mark.parametrize("M,N,K", [(3, 40, 700), (130, 200, 300), (300, 520, 1024)])
def test_not_finite_entries_stay_in_their_row_and_column(M, N, K):
    torch, dev = torch_dev()
    rng = np.random.default_rng(9)
    x, w = rng.standard_normal((M, K)).astype(np.float32), rng.standard_normal((N, K)).astype(np.float32)
    x[1, K // 2] = np.nan
    w[7, 3] = np.inf
    a, b = T.Blocks.empty(M, K), T.Blocks.empty(N, K)
    T.quantize_blocks(torch.from_numpy(x).to(dev), rows=a)
    T.quantize_blocks(torch.from_numpy(w).to(dev), rows=b)
    bad = np.zeros((M, N), dtype=bool)
    bad[1], bad[:, 7] = True, True
    out, _ = out_buffer(M, N, "bf16")
    T.matmul_blocks(a, b, out, workspace(M, N, K))
    np.testing.assert_array_equal(np.isnan(out.float().cpu().numpy()), bad)
    T.linear_blocks(torch.from_numpy(x).to(dev), b, out, workspace(M, N, K, True))
    np.testing.assert_array_equal(np.isnan(out.float().cpu().numpy()), bad)


@pytest.mark.parametrize("lo,hi", [(1, 3), (240, 248)])
def test_matmul_scales_at_both_ends(lo, hi):
    """The smallest and largest scales that quantising gives, against ones that bring the product back."""
    rng = np.random.default_rng(4)
    a, b = random_blocks(rng, 70, 400, "e4m3", lo, hi), random_blocks(rng, 90, 400, "e4m3", 254 - hi, 254 - lo)
    out, _ = out_buffer(70, 90, "f32")
    T.matmul_blocks(a, b, out, workspace(70, 90, 400))
    check_product(out.double().cpu().numpy(), values(a), values(b), "f32")


def test_matmul_offsets_beyond_32_bits():
    """Codes of more than 2^32 bytes and an output of more than 2^32: the last rows are right."""
    torch, dev = torch_dev()
    rng = np.random.default_rng(6)
    M, N, K = (1 << 21) + 70, 600, 2100
    b = random_blocks(rng, N, K, "e4m3")
    ld = O.up(K, 128)
    codes = torch.zeros((M, ld), dtype=torch.uint8, device=dev)
    scales = torch.full((-(-ld // 512), M, 4), 127, dtype=torch.uint8, device=dev)
    tail = random_blocks(rng, 100, K, "e4m3")
    codes[-100:] = tail.codes.view(torch.uint8)
    scales[:, -100:] = tail.scales
    a = T.Blocks(codes.view(torch.float8_e4m3fn), scales, K)
    out = torch.full((M, N), 7.0, dtype=torch.float32, device=dev)
    T.matmul_blocks(a, b, out, workspace(M, N, K))
    check_product(out[-100:].double().cpu().numpy(), values(tail), values(b), "f32")
    assert bool((out[:-100] == 0).all())
    del out
    x = torch.zeros((M, K), dtype=torch.bfloat16, device=dev)          # and a matrix of more than 2^32 bytes
    x[-3:] = torch.from_numpy(rng.standard_normal((3, K)).astype(np.float32)).to(dev)
    r, c = T.Blocks.empty(M, K), T.Blocks.empty(K, M)
    T.quantize_blocks(x, rows=r, cols=c)
    (codes, k), _ = O.quantize(x[-3:].double().cpu().numpy(), "e4m3")
    np.testing.assert_array_equal(host8(r.codes[-3:]), codes)
    np.testing.assert_array_equal(host8(r.scales[:, -3:]), O.lay_scales(k))
    tail_rows = M % 128
    _, (codes, _) = O.quantize(x[-tail_rows:].double().cpu().numpy(), "e4m3")
    np.testing.assert_array_equal(host8(c.codes[:, -128:]), codes)
    assert not host8(r.codes[:1000]).any() and not host8(c.codes[-1, :-128]).any()


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("name,out_name", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_linear_matches_oracle(M, N, K, name, out_name):
    rng = np.random.default_rng(M + N + K)
    x, xv = device(wild(rng, M, K) if M % 2 else rng.standard_normal((M, K)), name, shift=M % 3, pad=N % 4)
    w = random_blocks(rng, N, K, "e4m3" if N % 2 else "e5m2")
    (codes, k), _ = O.quantize(xv, "e4m3")
    A = O.matrix(codes, O.lay_scales(k), "e4m3")
    out, buf = out_buffer(M, N, out_name, pad=3, shift=1)
    T.linear_blocks(x, w, out, workspace(M, N, K, True))
    check_product(out.double().cpu().numpy(), A, values(w), out_name)
    whole = buf.double().cpu().numpy()
    beside = np.ones(whole.shape, dtype=bool)
    for m in range(M):
        beside[1 + m * (N + 3):1 + m * (N + 3) + N] = False
    assert (whole[beside] == 7.0).all()


@pytest.mark.parametrize("M,N,K", [(32, 70, 384), (19, 300, 600), (24, 4096, 512), (24, 4097, 512), (16, 4096, 700),
                                   (9, 4097, 900), (8, 4097, 1024), (32, 40, 385), (17, 33, 1)])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_linear_of_a_few_tokens_matches_oracle(M, N, K, name):
    rng = np.random.default_rng(M + N + K)
    x, xv = device(rng.standard_normal((M, K)) * 2.0 ** rng.integers(-20, 20, (M, 1)), name, shift=1, pad=2)
    w = random_blocks(rng, N, K, "e4m3")
    (codes, k), _ = O.quantize(xv, "e4m3")
    out, _ = out_buffer(M, N, "f32")
    T.linear_blocks(x, w, out, workspace(M, N, K, True), fast_sums=True)
    check_product(out.double().cpu().numpy(), O.matrix(codes, O.lay_scales(k), "e4m3"), values(w), "f32")


def test_products_repeat_their_bits():
    torch, dev = torch_dev()
    rng = np.random.default_rng(8)
    for M, N, K in ((1, 500, 4000), (40, 300, 3000), (256, 256, 8192), (700, 600, 1000)):
        a, b = random_blocks(rng, M, K, "e4m3"), random_blocks(rng, N, K, "e4m3")
        got = []
        for k in range(6):
            out, _ = out_buffer(M, N, "f32")
            T.matmul_blocks(a, b, out, workspace(M, N, K), fast_sums=k % 2 == 1)
            got.append(out.clone())
        assert all(torch.equal(got[k], got[k % 2]) for k in range(6))


def test_linear_layer_gradients():
    """y = x W^T, dX = dY W, dW = dY^T X through the products, on values that
    the format holds exactly: the formulas' results to the bit, and the
    differences of the loss sum(y dY) in x and W."""
    torch, dev = torch_dev()
    rng = np.random.default_rng(12)
    M, N, K = 150, 90, 200
    x, w, dy = (rng.integers(-4, 5, s).astype(np.float64) for s in ((M, K), (N, K), (M, N)))

    def forms(a, tile=False, fmt="e4m3"):
        r, c = T.Blocks.empty(*a.shape, fmt), T.Blocks.empty(*a.shape[::-1], fmt)
        T.quantize_blocks(torch.from_numpy(a.astype(np.float32)).to(dev), rows=r, cols=c, tile=tile)
        return r, c

    def product(a, b):
        out = torch.zeros((a.rows, b.rows), device=dev)
        T.matmul_blocks(a, b, out, workspace(a.rows, b.rows, a.cols))
        return out.double().cpu().numpy()

    (xr, xc), (wr, wc), (gr, gc) = forms(x), forms(w, True), forms(dy, fmt="e5m2")
    dx, dw = product(gr, wc), product(gc, xc)
    np.testing.assert_array_equal(product(xr, wr), x @ w.T)
    np.testing.assert_array_equal(dx, dy @ w)
    np.testing.assert_array_equal(dw, dy.T @ x)

    def loss(x, w):
        return (product(forms(x)[0], forms(w, True)[0]) * dy).sum()

    base = loss(x, w)
    for i, j in ((0, 0), (149, 199), (77, 131)):
        moved = x.copy()
        moved[i, j] += 1.0                               # linear: a difference of any length is the derivative
        assert loss(moved, w) - base == dx[i, j]
    for i, j in ((0, 0), (89, 199), (40, 128)):
        moved = w.copy()
        moved[i, j] += 1.0
        assert loss(x, moved) - base == dw[i, j]


# --- norm -----------------------------------------------------------------------------

LENGTHS = [1, 2, 7, 8, 127, 128, 129, 2047, 2048, 2049, 16385, 100003]


def gradients(rng, lengths=LENGTHS, scale=1.0):
    """Tensors of both types at odd addresses, and their values."""
    made = [device(rng.standard_normal(n) * scale, "bf16" if i % 3 == 1 else "f32", shift=i % 4) for i, n in enumerate(lengths)]
    return [t for t, _ in made], [v for _, v in made]


@pytest.mark.parametrize("scale", [1.0, 1e-30, 1e30])
@pytest.mark.parametrize("max_norm", [math.inf, 1.0, 1e-3])
def test_norm_matches_oracle(scale, max_norm):
    torch, dev = torch_dev()
    tensors, vals = gradients(np.random.default_rng(1), scale=scale)
    clip = torch.zeros(2, device=dev)
    T.grad_norm(T.GradSet(tensors), clip, grad_scale=0.25, max_norm=max_norm)
    n, f = O.norm(vals, 0.25, max_norm)
    got = clip.double().cpu().numpy()
    # the sums are in 64 bits: one rounding to fp32, and n 2^-53 of the sum
    assert abs(got[0] - n) <= 2 * U32 * n and abs(got[1] - f) <= 2 * U32 * f


def test_norm_of_nothing_and_of_what_is_not_finite():
    torch, dev = torch_dev()
    clip = torch.full((2,), 5.0, device=dev)
    T.grad_norm(T.GradSet([torch.zeros(0, device=dev)]), clip, max_norm=1.0)
    assert clip.tolist() == [0.0, 1.0]
    g = torch.ones(5000, device=dev)
    s = T.GradSet([g])
    for bad in (math.inf, -math.inf, math.nan):
        g[4999] = bad
        T.grad_norm(s, clip, max_norm=1.0)
        assert not math.isfinite(clip[0].item())
    g[4999] = 1.0
    T.grad_norm(s, clip, max_norm=1.0)
    assert clip[0].item() == np.float32(math.sqrt(5000.0))


def test_norm_of_many_workgroups_repeats_its_bits():
    torch, dev = torch_dev()
    g = torch.randn(30_000_001, device=dev)
    s = T.GradSet([g[:11], g[11:20_000_000], g[20_000_000:]])
    got = []
    for _ in range(5):
        clip = torch.zeros(2, device=dev)
        T.grad_norm(s, clip, max_norm=3.0)
        got.append(clip.tolist())
    n = math.sqrt(g.double().square().sum().item())
    assert all(v == got[0] for v in got) and abs(got[0][0] - n) <= 2 * U32 * n


# --- AdamW ------------------------------------------------------------------------------

def adamw_problem(rng, ptype, gtype, copies, lengths=LENGTHS):
    """Parameters and gradients of `lengths` at odd addresses, with their decay and rate factors."""
    torch, dev = torch_dev()
    p = [device(rng.standard_normal(n) * 0.02, ptype, shift=(i + 1) % 3)[0] for i, n in enumerate(lengths)]
    g = [device(rng.standard_normal(n) * 1e-3, gtype, shift=i % 3)[0] for i, n in enumerate(lengths)]
    cp = [device(np.zeros(n), "bf16", shift=i % 2)[0] for i, n in enumerate(lengths)] if copies else None
    wd = [0.1 * (i % 2) for i in range(len(lengths))]
    ls = [1.0 if i % 3 else 0.5 for i in range(len(lengths))]
    return p, g, cp, wd, ls


def vec(t):
    return t.double().cpu().numpy().ravel()


def state_values(codes, scale, fmt):
    k = np.repeat(host8(scale).astype(float) - 127, 128)[:codes.numel()]
    return O.code_values(fmt)[host8(codes).ravel()] * 2.0 ** k


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("ptype,gtype,copies", [("f32", "f32", True), ("f32", "bf16", False), ("bf16", "f32", False),
                                                ("bf16", "bf16", True)])
def test_adamw_matches_oracle(bits, ptype, gtype, copies):
    """Four steps, each checked from the state before it.  fp32 carries a
    handful of roundings a step; a code may differ from the oracle's only by
    one neighbour, where the chance falls within fp32's error of the limit: of
    the 4.9e5 entries checked, 2^-17 or so."""
    torch, dev = torch_dev()
    rng = np.random.default_rng(bits + copies)
    p, g, cp, wd, ls = adamw_problem(rng, ptype, gtype, copies)
    s = T.TensorSet(p, g, state_bits=bits, copies=cp, lr_scale=ls, weight_decay=wd)
    clip = torch.zeros(2, device=dev)
    places = np.concatenate([[0], np.cumsum([O.up(n, 128) for n in LENGTHS])])
    off = 0
    for step in range(1, 5):
        for t in g:
            t.copy_(torch.from_numpy((rng.standard_normal(t.numel()) * 1e-3).astype(np.float32)))
        T.grad_norm(s, clip, grad_scale=0.125, max_norm=0.01)
        factor = 0.125 * clip[1].item()
        before = []
        for i in range(len(p)):
            if bits == 32:
                m, v = vec(s.states["m"][i]), vec(s.states["v"][i])
            else:
                m = state_values(s.states["m"][i], s.states["m_scale"][i], "e4m3")
                v = state_values(s.states["v"][i], s.states["v_scale"][i], "e5m2")
            before.append((vec(p[i]), vec(g[i]), m, v))
        T.adamw_step(s, step, 1e-3, grad_scale=0.125, clip=clip, seed=77)
        for i, (p0, g0, m0, v0) in enumerate(before):
            p1, m1, v1 = O.adamw(p0, g0, m0, v0, step, 1e-3 * ls[i], 0.9, 0.999, 1e-8, wd[i], factor)
            got = vec(p[i])
            tol = 16 * U32 * (np.abs(p0) + np.abs(p1 - p0)) + 1e-12
            if ptype == "bf16":
                tol = tol + 2.0 ** -8 * np.abs(p1)
            assert (np.abs(got - p1) <= tol).all()
            if copies:
                assert torch.equal(cp[i], p[i].to(torch.bfloat16))
            if bits == 32:
                # g gs, its square, two products and the sum: six roundings of terms that may cancel
                assert (np.abs(vec(s.states["m"][i]) - m1) <= 8 * U32 * (0.9 * np.abs(m0) + 0.1 * np.abs(g0 * factor))).all()
                assert (np.abs(vec(s.states["v"][i]) - v1) <= 8 * U32 * v1 + 2.0 ** -149).all()
                continue
            rm, rv = O.chances(len(p0), int(places[i]), 77, step)
            for name, fmt, x, r in (("m", "e4m3", m1, rm), ("v", "e5m2", v1, rv)):
                codes, k = O.round_by_chance(x, fmt, r)
                np.testing.assert_array_equal(host8(s.states[name + "_scale"][i]), k + 127)
                diff = host8(s.states[name][i]).ravel().astype(int) - codes
                assert (np.abs(diff) <= 1).all()
                off += int((diff != 0).sum())
    # 16 fp32 units of error against spacings of 2^20 or more of them, both states, all entries
    assert off <= 30, off


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_step_without_a_finite_norm_changes_nothing(bits):
    torch, dev = torch_dev()
    rng = np.random.default_rng(2)
    p, g, cp, wd, ls = adamw_problem(rng, "f32", "f32", True, [300, 5])
    s = T.TensorSet(p, g, state_bits=bits, copies=cp)
    clip = torch.zeros(2, device=dev)
    T.adamw_step(s, 1, 1e-3)
    g[1][4] = math.nan
    T.grad_norm(s, clip)
    held = p + cp + [t for v in s.states.values() for t in v]
    before = [t.clone().view(torch.uint8) for t in held]
    T.adamw_step(s, 2, 1e-3, clip=clip)
    assert all(torch.equal(t.view(torch.uint8), b) for t, b in zip(held, before))
    g[1][4] = 0.0
    T.grad_norm(s, clip)
    T.adamw_step(s, 2, 1e-3, clip=clip)
    assert not torch.equal(p[0].view(torch.uint8).view(-1), before[0].view(-1))


def test_adamw_8_bit_averages_move_and_do_not_vanish():
    """Constant gradients: the stored averages approach g and g^2 although each
    step moves them by less than a code's spacing; and a square once seen is
    not forgotten to zero while the gradient rests."""
    torch, dev = torch_dev()
    n = 1280
    p, g = torch.zeros(n, device=dev), torch.full((n,), 0.5, device=dev)
    s = T.TensorSet([p], [g], state_bits=8)
    for step in range(1, 2001):
        T.adamw_step(s, step, 0.0, seed=3)
    m = state_values(s.states["m"][0], s.states["m_scale"][0], "e4m3")
    v = state_values(s.states["v"][0], s.states["v_scale"][0], "e5m2")
    # E[v] = (1 - 0.999^2000) g^2 = 0.8648 g^2; a code's spacing is 1/4 of it, and the average over
    # 1280 entries of a walk that stays within a few spacings is within 5 percent of that
    assert abs(m.mean() - 0.5) < 0.025 and abs(v.mean() - 0.8648 * 0.25) < 0.05 * 0.25
    g[:640] = 0.0
    g[640:] = 2.0 ** -40
    g[0:640:128] = 1e3
    g[1] = 2.0 ** -30
    for step in range(2001, 2101):
        T.adamw_step(s, step, 0.0, seed=3)
    assert (host8(s.states["v"][0]) != 0).all()


def test_adamw_8_bit_infinite_gradients_mark_their_own_entries():
    torch, dev = torch_dev()
    p, g = torch.ones(300, device=dev), torch.full((300,), 1e-2, device=dev)
    g[5], g[200] = math.inf, math.nan
    s = T.TensorSet([p], [g], state_bits=8)
    T.adamw_step(s, 1, 1e-3)
    bad = np.zeros(300, dtype=bool)
    bad[[5, 200]] = True
    for name, fmt in (("m", "e4m3"), ("v", "e5m2")):
        np.testing.assert_array_equal(~np.isfinite(state_values(s.states[name][0], s.states[name + "_scale"][0], fmt)), bad)
    np.testing.assert_array_equal(~np.isfinite(vec(p)), bad)


def test_adamw_8_bit_squares_far_below_their_block_stay_above_zero():
    torch, dev = torch_dev()
    g = torch.zeros(256, device=dev)
    g[0], g[1], g[2] = 1e15, 1e-15, 1.5e-19         # squares of 1e30, and of 1e-30 and 2.25e-38, which it dwarfs
    s = T.TensorSet([torch.zeros(256, device=dev)], [g], 8)
    T.adamw_step(s, 1, 1e-3, beta2=0.0)
    codes = host8(s.states["v"][0])
    assert codes[1] == 1 and codes[2] == 1 and codes[0] >= 0x78 and not codes[3:].any()


def test_adamw_8_bit_squares_beyond_fp32_are_infinite_as_32_bit_ones_are():
    """Finite gradients whose square passes 2^128: the second average is infinite and the
    step zero, for 8-bit states as for 32-bit ones, at this step and at later ones."""
    torch, dev = torch_dev()
    n, huge = 300, {3: 1e21, 5: -1e21, 130: 1.7e22, 131: 1e25, 260: -1e30, 299: 3e38}
    p, g = [], torch.full((n,), 1e-2, device=dev)
    for i, x in huge.items():
        g[i] = x
    at, rest = list(huge), [i for i in range(n) if i not in huge]
    for bits in (32, 8):
        q = torch.linspace(1.0, 2.0, n, device=dev)
        start = q.clone()
        s = T.TensorSet([q], [g], state_bits=bits)
        for step in range(1, 4):
            T.adamw_step(s, step, 1e-3, seed=step)
            assert torch.equal(q[at], start[at]) and bool(torch.isfinite(q).all())
            if step == 1:
                p.append(q[rest].clone())
        m, v = s.states["m"][0].double(), s.states["v"][0].double()
        assert bool(torch.isfinite(m).all()) and bool(torch.isinf(v[at]).all()) and bool(torch.isfinite(v[rest]).all())
    # the first step is of 1e-3 from exact states of zero: fp32's 24 bits against 24 bits cut off, then the parameter's rounding
    assert (p[0] - p[1]).abs().max().item() <= 8 * U32 * 1e-3 + 2 * U32 * 2


def test_adamw_8_bit_states_below_the_normal_numbers():
    """Averages of 2^-136 to 2^-122, in blocks whose scale is the smallest: the oracle's
    codes.  fp32 holds a number of 2^-136 to 2^-14 of it, a code's spacing is an eighth or
    more of a number: of the 1024 entries one or two may fall on the neighbour."""
    torch, dev = torch_dev()
    rng = np.random.default_rng(21)
    for name, fmt, g in (("v", "e5m2", 2.0 ** rng.uniform(-68, -61, 1024)), ("m", "e4m3", 2.0 ** rng.uniform(-125, -119, 1024))):
        t, g = device(g)
        s = T.TensorSet([torch.zeros(1024, device=dev)], [t], state_bits=8)
        # beta2 = 0 and beta1 = 0.875: v = g^2 and m = g / 8, exact in fp64
        T.adamw_step(s, 1, 1e-3, beta1=0.875, beta2=0.0, seed=5)
        r = dict(zip("mv", O.chances(1024, 0, 5, 1)))[name]
        codes, k = O.round_by_chance(g * g if name == "v" else g / 8, fmt, r)
        np.testing.assert_array_equal(host8(s.states[name + "_scale"][0]), k + 127)
        diff = host8(s.states[name][0]).astype(int) - codes
        assert (np.abs(diff) <= 1).all() and (diff != 0).sum() <= 2, (name, (diff != 0).sum())


def test_norm_beyond_fp32_is_infinite_and_nothing_is_stepped():
    torch, dev = torch_dev()
    g = torch.full((5000,), 3e38, device=dev)
    p = torch.ones(5000, device=dev)
    s = T.TensorSet([p], [g])
    clip = torch.zeros(2, device=dev)
    T.grad_norm(s, clip, max_norm=1.0)
    assert clip[0].item() == math.inf
    T.adamw_step(s, 1, 1e-3, clip=clip)
    assert (p == 1).all() and not s.states["m"][0].any() and not s.states["v"][0].any()
    T.grad_norm(s, clip, grad_scale=1e-3, max_norm=1.0)
    assert clip[0].item() == pytest.approx(3e35 * math.sqrt(5000), rel=1e-6)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_many_small_and_one_large_tensor(bits):
    """Thousands of pieces: the step over all tensors equals the steps of each alone (32 bits)
    and repeats its bits (8)."""
    torch, dev = torch_dev()
    lengths = [3] * 300 + [9_000_001] + [700] * 40
    gen = torch.Generator(device=dev).manual_seed(1)

    def made():
        gen.manual_seed(1)
        return ([torch.randn(n, device=dev, generator=gen) for n in lengths],
                [torch.randn(n, device=dev, generator=gen) for n in lengths])

    p, g = made()
    T.adamw_step(T.TensorSet(p, g, state_bits=bits, weight_decay=0.1), 1, 1e-2, seed=5)
    q, g = made()
    if bits == 32:
        for a, b in zip(q, g):
            T.adamw_step(T.TensorSet([a], [b], weight_decay=0.1), 1, 1e-2)
            torch.cuda.synchronize()
    else:
        T.adamw_step(T.TensorSet(q, g, state_bits=8, weight_decay=0.1), 1, 1e-2, seed=5)
    assert all(torch.equal(a, b) for a, b in zip(p, q))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("lr,wd", [(1e-5, 0.05), (2.5e-6, 0.01)])
def test_adamw_small_decays_add_up(bits, lr, wd):
    """Two runs of 400 steps on the same gradients, one with decay: without rounding,
    their parameters part by lr wd times the sum of the decayed run's parameters.
    A step rounds a parameter of 0.5 to 1 by 2^-25 at most, at random: the updates
    of the two runs are of 40 to 170 units in the last place and new at every step.  Over
    400 steps and 65536 entries the mean of the two walks is within 6 sqrt(2) 2^-25
    sqrt(400 / (3 * 65536)) = 1.2e-8; the decays are 1.5e-4 and 7.5e-6 in all."""
    torch, dev = torch_dev()
    n, steps = 1 << 16, 400
    gen = torch.Generator(device=dev).manual_seed(1)
    start = 0.5 + 0.5 * torch.rand(n, device=dev, generator=gen)
    p, g = [start.clone(), start.clone()], torch.zeros(n, device=dev)
    sets = [T.TensorSet([q], [g], state_bits=bits, weight_decay=d) for q, d in zip(p, (wd, 0.0))]
    total = torch.zeros((), dtype=torch.float64, device=dev)
    for step in range(1, steps + 1):
        g.normal_(generator=gen)
        total += p[0].double().mean()
        for s in sets:
            T.adamw_step(s, step, lr, seed=2)
    parted = (p[1].double() - p[0].double()).mean().item()
    assert abs(parted - lr * wd * total.item()) <= 5e-8


def test_sets_refuse_on_the_device():
    torch, dev = torch_dev()
    p, g = torch.zeros(10, device=dev), torch.zeros(10, device=dev)
    with pytest.raises(C.CerarError, match="overlap"):
        T.TensorSet([p, p], [g, g])
    with pytest.raises(ValueError, match="entries"):
        T.TensorSet([p], [g[:9]])
    with pytest.raises(ValueError, match="contiguous"):
        T.TensorSet([p], [torch.zeros(20, device=dev)[::2]])
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        T.TensorSet([p.half()], [g])
    with pytest.raises(ValueError, match="states must hold"):
        T.TensorSet([p], [g], states={"m": [p]})
    s = T.GradSet([g])
    with pytest.raises(C.CerarError, match="gradients alone"):
        T.adamw_step(s, 1, 1e-3)
    clip = torch.zeros(2, device=dev)
    for kw in ({"grad_scale": 0.0}, {"grad_scale": math.inf}, {"max_norm": 0.0}, {"max_norm": math.nan}):
        with pytest.raises(C.CerarError):
            T.grad_norm(s, clip, **kw)
    with pytest.raises(ValueError, match="clip"):
        T.grad_norm(s, torch.zeros(1, device=dev))
    s = T.TensorSet([p], [g])
    for kw in ({}, {"step": 1}, {"step": 1, "lr": 1e-3, "values": torch.zeros(64, dtype=torch.uint8, device=dev)}):
        with pytest.raises(ValueError):
            T.adamw_step(s, **kw)
    x, w = torch.zeros((4, 300), device=dev), T.Blocks.empty(6, 300)
    with pytest.raises(ValueError, match="out has shape"):
        T.linear_blocks(x, w, torch.zeros((4, 7), device=dev), workspace(4, 6, 300, True))
    with pytest.raises(ValueError, match="row-major"):
        T.linear_blocks(x.t().contiguous().t(), w, torch.zeros((4, 6), device=dev), workspace(4, 6, 300, True))
    with pytest.raises(C.CerarError, match="by_row is"):
        T.quantize_blocks(x, rows=w)
    with pytest.raises(C.CerarError, match="columns"):
        T.matmul_blocks(w, T.Blocks.empty(6, 301), torch.zeros((6, 6), device=dev))


@pytest.mark.parametrize("bits", [32, 8])
def test_a_backward_that_saved_what_a_step_wrote_raises(bits):
    """Parameters and their copies count the step's writes, whether they are tensors of
    their own or views of one; a step that is refused counts nothing."""
    torch, dev = torch_dev()
    flat = torch.ones(600, device=dev)
    p = [torch.nn.Parameter(torch.ones(200, device=dev)), flat[:300].view(20, 15), flat[300:]]
    g = [torch.full_like(t, 1e-2) for t in p]
    cp = [torch.zeros_like(t, dtype=torch.bfloat16) for t in p]
    s = T.TensorSet([t.detach() if t.requires_grad else t for t in p], g, state_bits=bits, copies=cp)
    x = torch.ones((), device=dev, requires_grad=True)

    def losses():
        return [t.square().sum() if t.requires_grad else (x * t).sum() for t in p + cp]

    for loss in losses():
        loss.backward()                                  # none has been written since
    saved = losses()
    with pytest.raises(C.CerarError):
        T.adamw_step(s, 0, 1e-3)
    saved.pop(0).backward()
    saved = losses()
    T.adamw_step(s, 1, 1e-3)
    for loss in saved:
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    for loss in losses():
        loss.backward()
    T.adamw_step(s, values=T.adamw_values(2, 1e-3).to(dev))
    assert [t._version for t in s._stepped] == [2] * len(s._stepped)


def test_a_backward_that_saved_a_product_raises_once_it_is_overwritten():
    torch, dev = torch_dev()
    a, w = T.Blocks.empty(5, 300), T.Blocks.empty(6, 300)
    v = torch.ones((5, 300), device=dev)
    T.quantize_blocks(v, rows=a)
    T.quantize_blocks(torch.ones((6, 300), device=dev), rows=w)
    x, out = torch.ones((), device=dev, requires_grad=True), torch.zeros((5, 6), device=dev)
    for call in (lambda: T.matmul_blocks(a, w, out), lambda: T.matmul_blocks(a, w, out, accumulate=True),
                 lambda: T.linear_blocks(v, w, out, workspace(5, 6, 300, True))):
        (x * out).sum().backward()
        loss = (x * out).sum()
        call()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()


def test_inference_tensors_are_stepped_and_written():
    torch, dev = torch_dev()
    with torch.inference_mode():
        p, g = torch.ones(10, device=dev), torch.ones(10, device=dev)
        s = T.TensorSet([p[:4], p[4:]], [g[:4], g[4:]])
        T.adamw_step(s, 1, 1e-3)
        assert bool((p < 1).all())
        w = T.Blocks.empty(6, 300)
        T.quantize_blocks(torch.ones((6, 300), device=dev), rows=w)
        out = torch.zeros((1, 6), device=dev)
        T.linear_blocks(torch.ones((1, 300), device=dev), w, out, workspace(1, 6, 300, True))
        assert bool((out == 300).all())


# --- streams and graphs --------------------------------------------------------------------

class Problem:
    """A layer's products, norm and step on buffers that stay in place."""

    def __init__(self, bits, seed=1):
        torch, dev = torch_dev()
        self.M, self.N, self.K = 70, 200, 300
        gen = torch.Generator(device=dev).manual_seed(seed)
        self.x = torch.randn((self.M, self.K), device=dev, generator=gen)
        self.dy = torch.randn((self.M, self.N), device=dev, generator=gen)
        self.w = torch.randn((self.N, self.K), device=dev, generator=gen) * 0.1
        self.grad = torch.zeros_like(self.w)
        self.y = torch.zeros((self.M, self.N), dtype=torch.bfloat16, device=dev)
        self.token = torch.zeros((1, self.N), device=dev)
        self.wr, self.xc = T.Blocks.empty(self.N, self.K), T.Blocks.empty(self.K, self.M)
        self.xr, self.gc = T.Blocks.empty(self.M, self.K), T.Blocks.empty(self.N, self.M, "e5m2")
        self.clip = torch.zeros(2, device=dev)
        self.set = T.TensorSet([self.w], [self.grad], state_bits=bits)
        self.ws = [workspace(self.M, self.N, self.K), workspace(self.N, self.K, self.M), workspace(1, self.N, self.K, True)]
        self.values = T.adamw_values(1, 1e-2, seed=4).to(dev)

    def step(self, stream=None):
        T.quantize_blocks(self.w, rows=self.wr, tile=True, stream=stream)
        T.quantize_blocks(self.x, rows=self.xr, cols=self.xc, stream=stream)
        T.quantize_blocks(self.dy, cols=self.gc, stream=stream)
        T.matmul_blocks(self.xr, self.wr, self.y, self.ws[0], stream=stream)
        T.matmul_blocks(self.gc, self.xc, self.grad, self.ws[1], accumulate=True, stream=stream)
        T.linear_blocks(self.x[:1], self.wr, self.token, self.ws[2], stream=stream)
        T.grad_norm(self.set, self.clip, max_norm=1.0, stream=stream)
        T.adamw_step(self.set, clip=self.clip, values=self.values, stream=stream)

    def results(self):
        torch, _ = torch_dev()
        return [t.clone().view(torch.uint8) for t in (self.y, self.token, self.grad, self.clip, self.w,
                                                      self.set.states["m"][0], self.set.states["v"][0])]


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_step_replays(bits):
    """A step recorded into a graph and replayed with the next step's values
    copied in, beside the same steps run eagerly, with eager work between."""
    torch, dev = torch_dev()
    a, b = Problem(bits), Problem(bits)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    torch.cuda.synchronize()
    for k in range(1, 5):
        for prob in (a, b):
            prob.values.copy_(T.adamw_values(k, 1e-2 / k, seed=4))
            prob.x.copy_(torch.from_numpy(np.random.default_rng(k).standard_normal((70, 300)).astype(np.float32)))
        graph.replay()
        b.step()
        torch.cuda.synchronize()
        for i, (u, v) in enumerate(zip(a.results(), b.results())):
            assert torch.equal(u, v), (k, i)
    del graph


def test_step_on_another_stream():
    torch, dev = torch_dev()
    a, b = Problem(32), Problem(32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        a.step(stream=side)
        b.step()
    torch.cuda.synchronize()
    for u, v in zip(a.results(), b.results()):
        assert torch.equal(u, v)


@pytest.mark.parametrize("bits", [32, 8])
def test_states_made_on_a_busy_stream_are_zero_before_a_step_on_another(bits):
    torch, dev = torch_dev()
    busy, other = torch.cuda.Stream(), torch.cuda.Stream()
    p, g = torch.ones(5000, device=dev), torch.ones(5000, device=dev)
    x, y = torch.ones((4096, 4096), device=dev), torch.empty((4096, 4096), device=dev)
    torch.cuda.synchronize()
    with torch.cuda.stream(busy):
        for _ in range(40):
            torch.mm(x, x, out=y)
        s = T.TensorSet([p], [g], state_bits=bits)
    T.adamw_step(s, 1, 1e-3, stream=other)
    torch.cuda.synchronize()
    assert bool((s.states["m"][0].float() != 0).all()) and bool((s.states["v"][0].float() != 0).all())


def test_values_equal_the_settings():
    torch, dev = torch_dev()
    out = []
    for use in (False, True):
        p, g = torch.linspace(-1, 1, 500, device=dev), torch.linspace(1, 2, 500, device=dev)
        s = T.TensorSet([p], [g])
        for k in range(1, 4):
            kw = dict(step=k, lr=1e-2, beta1=0.8, beta2=0.95, eps=1e-6, grad_scale=0.5)
            if use:
                T.adamw_step(s, values=T.adamw_values(**kw).to(dev))
            else:
                T.adamw_step(s, **kw)
        out.append(p)
    assert torch.equal(*out)
