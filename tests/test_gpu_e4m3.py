"""ks_quantize_e4m3 and ks_matmul_e4m3 against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

from tests import lowbit
from paper_2609_35587_b200 import binding as ks
from paper_2609_35587_b200 import workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx():
    c = ks.Context(wl.gpu_desc(), 0)
    yield c
    assert c.device_status() == ks.KS_OK
    c.close()


def values(rows, cols, seed, dtype=torch.float32):
    """Rows and blocks of very different size."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(3 * torch.randn(rows, 1, generator=g))
    x *= torch.exp2(2 * torch.randn(1, cols, generator=g))
    return x.to(dtype).to(DEV)


# ---- quantiser ----------------------------------------------------------------------------------


def check_quantized(q, s, x, block_rows, scale):
    want_q, want_s = lowbit.quantize(lowbit.as_float64(x), block_rows, scale)
    np.testing.assert_array_equal(lowbit.as_float64(s), want_s)
    np.testing.assert_array_equal(lowbit.as_float64(q), want_q)


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 127), (5, 128), (2, 129), (130, 300), (257, 1024), (1, 4099)])
def test_quantize(ctx, rows, cols, dtype, block_rows, scale):
    x = values(rows, cols, rows + cols, dtype)
    q, s = ctx.quantize_e4m3(x, block_rows=block_rows, scale=scale)
    check_quantized(q, s, x, block_rows, scale)


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_odd_values(ctx, block_rows, scale):
    """Zeros, numbers that are none, values at the borders of a scale and of the type."""
    x = torch.zeros(12, 512)
    x[0, :128] = torch.linspace(-448, 448, 128)
    x[1, 3], x[1, 130], x[1, 300] = 449.0, 448.0 * 2 ** 20, float(np.nextafter(np.float32(448), np.float32(500)))
    x[2, 5], x[2, 6], x[2, 7], x[2, 8] = np.inf, -np.inf, np.nan, 3.0
    x[3] = np.nan
    x[4, 0], x[4, 1] = 1e-45, -1e-45
    x[4, 128], x[4, 129] = 2.0 ** -126, 2.0 ** -140
    x[5, 0], x[5, 200] = 3.4028234663852886e38, -3.4028234663852886e38
    x[6, :256] = torch.exp2(torch.arange(256.0) / 16 - 8)
    x[7, 0], x[7, 1] = 2.0 ** -100, 2.0 ** -101
    x[8, :128] = torch.arange(128.0) / 64  # ties between neighbours
    x[8, 127] = 448.0
    x[9, 0], x[9, 1:128] = 448.0, 2.0 ** -10  # half of the smallest step
    x = x.to(DEV)
    q, s = ctx.quantize_e4m3(x, block_rows=block_rows, scale=scale)
    check_quantized(q, s, x, block_rows, scale)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantize_leaves_what_is_not_its_own(ctx, dtype):
    """Strided and unaligned input rows; bytes behind a row's end and rows behind the last stay as they were."""
    big = values(40, 777, 3, dtype)
    x = big[2:35, 1:300]  # 33 rows of 299, odd offset
    out = torch.full((35, 320), 0x55, dtype=torch.uint8, device=DEV)
    scales = torch.full((35, 3), 0x55, dtype=torch.uint8, device=DEV)
    q, s = ctx.quantize_e4m3(x, out=out.view(torch.float8_e4m3fn)[:33, :299], out_scale=scales[:33].view(torch.float8_e8m0fnu))
    check_quantized(q, s, x, 1, "e8m0")
    assert bool((out[:33, 299:] == 0x55).all()) and bool((out[33:] == 0x55).all()) and bool((scales[33:] == 0x55).all())


# ---- product ------------------------------------------------------------------------------------


def operands(m, n, k, scale, seed):
    """Quantised by the definition, not by the kernel."""
    def one(x, block_rows):
        q, s = lowbit.quantize(lowbit.as_float64(x), block_rows, scale)
        qt = torch.zeros(x.shape[0], -(-max(x.shape[1], 1) // 16) * 16)
        qt[:, :x.shape[1]] = torch.from_numpy(q)
        dt = torch.float8_e8m0fnu if scale == "e8m0" else torch.float32
        return qt.to(torch.float8_e4m3fn).to(DEV)[:, :x.shape[1]], torch.from_numpy(s).float().to(dt).to(DEV), q, s
    return one(values(m, k, seed), 1), one(values(n, k, seed + 1), 128)


def off_by(k, mag, want, dtype):
    """What fp32 sums and one rounding may lose: at most k + blocks + 4 additions or products, each off by 2^-23 of the
    magnitudes' sum (an addition that truncates; one that rounds loses half), then half a step of the result's type, or of
    its smallest numbers."""
    t = (k + lowbit.blocks_of(k) + 4) * 2.0 ** -23 * mag
    if dtype == torch.float32:
        return t + 2.0 ** -24 * np.abs(want)
    half = torch.finfo(dtype).eps / 2
    return t * (1 + half) + half * np.abs(want) + (2.0 ** -25 if dtype == torch.float16 else 0.0)


SHAPES = [(1, 1, 1), (1, 128, 128), (1, 1000, 4096), (7, 130, 129), (16, 512, 1000), (17, 64, 640), (33, 300, 77), (64, 384, 2048),
          (65, 129, 128), (128, 256, 256), (129, 255, 300), (200, 1024, 1024), (256, 512, 384), (300, 700, 500), (513, 257, 129),
          (1025, 1100, 520), (4200, 130, 300), (1300, 520, 2100), (2100, 520, 2100)]


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_matmul(ctx, m, n, k, scale):
    (a, sa, av, sav), (b, sb, bv, sbv) = operands(m, n, k, scale, m + n + k)
    want, mag = lowbit.matmul(av, sav, bv, sbv)
    got = ctx.matmul_e4m3(a, sa, b, sb, out_dtype=torch.float32)
    err = np.abs(lowbit.as_float64(got) - want)
    assert (err <= off_by(k, mag, want, torch.float32)).all(), err.max()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m,n,k", [(1, 300, 256), (48, 1000, 700), (100, 130, 256), (300, 500, 700), (4200, 130, 256), (1100, 600, 700)])
def test_matmul_epilogue(ctx, m, n, k, dtype):
    """Bias, ReLU, each result type, a result with padded rows of which nothing else is written."""
    (a, sa, av, sav), (b, sb, bv, sbv) = operands(m, n, k, "f32", 5)
    sum64, mag = lowbit.matmul(av, sav, bv, sbv)
    top = np.abs(sum64).max() + 1
    sa = sa / float(np.float32(top))  # the sums fit 16 bits
    sav = lowbit.as_float64(sa)
    sum64, mag = lowbit.matmul(av, sav, bv, sbv)
    bias = torch.linspace(-0.3, 0.3, n, device=DEV)
    out = torch.full((m + 2, n + 5), 7.0, dtype=dtype, device=DEV)
    for relu in (False, True):
        got = ctx.matmul_e4m3(a, sa, b, sb, bias=bias, relu=relu, out_dtype=dtype, out=out[:m, :n])
        want = sum64 + lowbit.as_float64(bias)
        if relu:
            want = np.maximum(want, 0)
        err = np.abs(lowbit.as_float64(got) - want)
        assert (err <= off_by(k, mag + np.abs(lowbit.as_float64(bias)), want, dtype)).all(), err.max()
        assert bool((out[m:] == 7).all()) and bool((out[:, n:] == 7).all())


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("m,n,k", [(1, 256, 256), (5, 129, 300), (64, 1000, 512), (130, 128, 128), (300, 450, 1024), (4200, 130, 300), (1200, 450, 1024)])
def test_matmul_quantised_result(ctx, m, n, k, scale):
    (a, sa, av, sav), (b, sb, bv, sbv) = operands(m, n, k, scale, 9)
    sums, mag = lowbit.matmul(av, sav, bv, sbv)
    want = np.maximum(sums, 0)
    wide = torch.full((m + 1, (n + 31) // 16 * 16), 0x55, dtype=torch.uint8, device=DEV)
    q, s = ctx.matmul_e4m3(a, sa, b, sb, relu=True, out_dtype=torch.float8_e4m3fn, out=wide.view(torch.float8_e4m3fn)[:m, :n])
    tol = off_by(k, mag, want, torch.float32)
    s64, q64 = lowbit.as_float64(s), lowbit.as_float64(q)
    # the scale is that of some maximum within the sums' tolerance
    amax, off = lowbit.block_amax(want, 1), lowbit.block_amax(tol, 1)
    if scale == "e8m0":
        assert ((lowbit.scale_e8m0(np.maximum(amax - off, 0)) <= s64) & (s64 <= lowbit.scale_e8m0(amax + off))).all()
    else:
        low = np.maximum(np.maximum(amax - off, 0), 2.0 ** -100) / 448 * (1 - 2.0 ** -23)
        assert ((low <= s64) & (s64 <= np.maximum(amax + off, 2.0 ** -100) / 448 * (1 + 2.0 ** -23))).all()
    per = np.repeat(s64, 128, 1)[:, :n]
    # half a step of three mantissa bits, or of the smallest; fp32 products in front of it
    assert (np.abs(q64 * per - want) <= tol + (2.0 ** -4 + 2.0 ** -22) * (want + tol) + 2.0 ** -10 * per).all()
    assert bool((wide[m:] == 0x55).all()) and bool((wide[:, n:] == 0x55).all())


@pytest.mark.parametrize("m", [3, 300, 4200])
@pytest.mark.parametrize("scale", [torch.float32, torch.float8_e8m0fnu])
def test_matmul_empty_sum_of_many_rows(ctx, m, scale):
    a, b = torch.empty(m, 0, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(130, 0, dtype=torch.float8_e4m3fn, device=DEV)
    bias = torch.arange(130.0, device=DEV) - 60
    sa, sb = (torch.empty(r, 0, device=DEV).to(scale) for r in (m, 2))
    got = ctx.matmul_e4m3(a, sa, b, sb, bias=bias, relu=True, out_dtype=torch.float32)
    assert torch.equal(got, bias.clamp(min=0).expand(m, 130))
    assert not bool(ctx.matmul_e4m3(a, sa, b, sb).any())


def test_matmul_empty_sum(ctx):
    a = torch.empty(3, 16, device=DEV).to(torch.float8_e4m3fn)[:, :0]
    s = torch.empty(3, 0, device=DEV)
    b = torch.empty(130, 16, device=DEV).to(torch.float8_e4m3fn)[:, :0]
    bias = torch.arange(130.0, device=DEV) - 60
    got = ctx.matmul_e4m3(a, s, b, torch.empty(2, 0, device=DEV), bias=bias, relu=True, out_dtype=torch.float32)
    assert torch.equal(got, bias.clamp(min=0).expand(3, 130))


@pytest.mark.parametrize("m", [3, 200, 4200])
@pytest.mark.parametrize("scale", ["e8m0", "f32"])
def test_matmul_not_a_number(ctx, m, scale):
    """A code that is no number spoils its row (a) or column (b) and nothing else; ReLU makes 0 of it."""
    (a, sa, av, sav), (b, sb, bv, sbv) = operands(m, 140, 300, scale, 4)
    a.view(torch.uint8)[2, 299] = 0x7F
    b.view(torch.uint8)[133, 5] = 0xFF
    want, mag = lowbit.matmul(av, sav, bv, sbv)
    got = lowbit.as_float64(ctx.matmul_e4m3(a, sa, b, sb, out_dtype=torch.float32))
    spoiled = np.zeros((m, 140), bool)
    spoiled[2], spoiled[:, 133] = True, True
    assert np.isnan(got[spoiled]).all()
    assert (np.abs(got - want) <= off_by(300, mag, want, torch.float32))[~spoiled].all()
    got = lowbit.as_float64(ctx.matmul_e4m3(a, sa, b, sb, relu=True, out_dtype=torch.float32))
    assert (got[spoiled] == 0).all()


@pytest.mark.parametrize("m", [40, 4200])
@pytest.mark.parametrize("scale", ["e8m0", "f32"])
def test_matmul_extreme_scales(ctx, scale, m):
    """Scales far from one whose product is an ordinary number."""
    (a, sa, av, sav), (b, sb, bv, sbv) = operands(m, 130, 260, scale, 8)
    up = torch.full_like(sa, 2.0 ** 60, dtype=torch.float32)
    sa, sb = (sa.float() * up).to(sa.dtype), (sb.float() * 2.0 ** -60).to(sb.dtype)
    want, mag = lowbit.matmul(av, sav, bv, sbv)
    got = ctx.matmul_e4m3(a, sa, b, sb, out_dtype=torch.float32)
    assert (np.abs(lowbit.as_float64(got) - want) <= off_by(260, mag, want, torch.float32)).all()


@pytest.mark.parametrize("m,n,k", [(1, 700, 1000), (300, 300, 400), (4200, 300, 400)])
def test_matmul_same_bits_in_streams_and_graphs(ctx, m, n, k):
    (a, sa, _, _), (b, sb, _, _) = operands(m, n, k, "e8m0", 6)
    first = ctx.matmul_e4m3(a, sa, b, sb)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(first)
    with torch.cuda.stream(side):
        ctx.matmul_e4m3(a, sa, b, sb, out=out)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, out)
    x = torch.zeros(m, k, device=DEV)
    q, s = ctx.quantize_e4m3(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.quantize_e4m3(x, out=q, out_scale=s)
        ctx.matmul_e4m3(q, s, b, sb, out=out)
    for seed in (1, 2):
        x.copy_(values(m, k, seed))
        graph.replay()
        q2, s2 = ctx.quantize_e4m3(x)
        assert torch.equal(out, ctx.matmul_e4m3(q2, s2, b, sb))


def test_matmul_long_sums(ctx):
    """Many blocks of K: several parts of an accumulator, several chunks of scales, ends inside both."""
    for m, n, k in ((130, 130, 4096 + 128 * 3 + 5), (20, 70, 20000), (257, 100, 12345), (2300, 515, 4096 + 200), (1030, 1030, 2600)):
        for scale in ("e8m0", "f32"):
            (a, sa, av, sav), (b, sb, bv, sbv) = operands(m, n, k, scale, 2)
            want, mag = lowbit.matmul(av, sav, bv, sbv)
            got = ctx.matmul_e4m3(a, sa, b, sb, out_dtype=torch.float32)
            assert (np.abs(lowbit.as_float64(got) - want) <= off_by(k, mag, want, torch.float32)).all()


@pytest.mark.parametrize("m", [30, 300, 4200])
def test_matmul_scale_that_is_no_number(ctx, m):
    """The byte 255 spoils its row's sums."""
    (a, sa, av, sav), (b, sb, bv, sbv) = operands(m, 140, 300, "e8m0", 4)
    sa.view(torch.uint8)[5, 1] = 255
    want, mag = lowbit.matmul(av, sav, bv, sbv)
    got = lowbit.as_float64(ctx.matmul_e4m3(a, sa, b, sb, out_dtype=torch.float32))
    assert np.isnan(got[5]).all()
    rest = np.arange(m) != 5
    assert (np.abs(got - want)[rest] <= off_by(300, mag, want, torch.float32)[rest]).all()


def test_two_graphs_and_an_eager_call(ctx):
    """Two captured products replayed in turn with a call in between: they share nothing."""
    sets = []
    for seed, m in ((1, 20), (2, 300), (3, 4200)):
        (a, sa, _, _), (b, sb, _, _) = operands(m, 200, 300, "e8m0", seed)
        out = ctx.matmul_e4m3(a, sa, b, sb)
        want = out.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ctx.matmul_e4m3(a, sa, b, sb, out=out)
        sets.append((graph, out, want, (a, sa, b, sb)))
    for _ in range(3):
        for graph, out, _, _ in sets:
            out.zero_()
            graph.replay()
        eager = ctx.matmul_e4m3(*sets[0][3])
        for _, out, want, _ in sets:
            assert torch.equal(out, want)
        assert torch.equal(eager, sets[0][2])


def test_binding_refuses(ctx):
    (a, sa, _, _), (b, sb, _, _) = operands(4, 8, 32, "f32", 1)
    with pytest.raises(ValueError):
        ctx.matmul_e4m3(a, sa[:, :0], b, sb)
    with pytest.raises(ValueError):
        ctx.matmul_e4m3(a.float(), sa, b, sb)
    with pytest.raises(ValueError):
        ctx.matmul_e4m3(a, sa, b, sb.to(torch.float8_e8m0fnu))
    with pytest.raises(ValueError):
        ctx.matmul_e4m3(a, sa, b[:, :16], sb)
    with pytest.raises(ValueError):
        ctx.matmul_e4m3(a, sa, b, sb, bias=torch.zeros(7, device=DEV))
    with pytest.raises(ValueError):
        ctx.quantize_e4m3(torch.zeros(4, 8, device=DEV)[:, ::2])
    with pytest.raises(ks.KsError):
        ctx.quantize_e4m3(torch.zeros(4, 4, device=DEV), block_rows=2)
    with pytest.raises(ks.KsError):  # rows that do not begin on 16-byte boundaries
        ctx.matmul_e4m3(torch.zeros(4, 20, device=DEV).to(torch.float8_e4m3fn), sa, torch.zeros(8, 20, device=DEV).to(torch.float8_e4m3fn), sb)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("m", [40, 300, 4200])
@pytest.mark.parametrize("ldd", [256, 264, 260, 257, 258])
def test_matmul_rows_that_begin_anywhere(ctx, m, ldd, dtype, scale):
    """Results whose rows begin on boundaries of 32 bytes, of 16 and of less, at the buffer's start and inside it."""
    n, k = 256, 200
    (a, sa, av, sav), (b, sb, bv, sbv) = operands(m, n, k, scale, 3)
    top = float(2.0 ** np.ceil(np.log2(np.abs(lowbit.matmul(av, sav, bv, sbv)[0]).max())))
    sa = (sa.float() / top).to(sa.dtype)  # the sums fit 16 bits
    want, mag = lowbit.matmul(av, lowbit.as_float64(sa), bv, sbv)
    for start in (0, 8, 3):
        flat = torch.full((m * ldd + 16,), 7.0, dtype=dtype, device=DEV)
        out = flat[start:start + m * ldd].view(m, ldd)[:, :n]
        ctx.matmul_e4m3(a, sa, b, sb, out_dtype=dtype, out=out)
        assert (np.abs(lowbit.as_float64(out) - want) <= off_by(k, mag, want, dtype)).all()
        left = flat.clone()
        left[start:start + m * ldd].view(m, ldd)[:, :n] = 7.0
        assert bool((left == 7).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("n,k", [(64, 64), (128, 256), (256, 80), (1024, 1024)])
def test_matmul_rows_by_themselves(ctx, n, k, dtype):
    """With powers of two and K up to 1,024 a row's result does not depend on the rows beside it."""
    m = 4500
    (a, sa, _, _), (b, sb, _, _) = operands(m, n, k, "e8m0", 11)
    values_of = lambda r: [t.view(torch.uint8) for t in r] if dtype == torch.float8_e4m3fn else [r]  # noqa: E731
    whole = values_of(ctx.matmul_e4m3(a, sa, b, sb, relu=True, out_dtype=dtype))
    for first, rows in ((0, 1), (4321, 1), (100, 16), (7, 17), (300, 60), (511, 130), (0, 1000), (255, 4097)):
        part = values_of(ctx.matmul_e4m3(a[first:first + rows], sa[first:first + rows], b, sb, relu=True, out_dtype=dtype))
        for w, p in zip(whole, part):
            assert torch.equal(w[first:first + rows], p), (first, rows)


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("m,n,k", [(8, 512, 2048), (100, 300, 256), (2300, 300, 256)])
def test_buffers_written_again_by_calls_that_follow_at_once(ctx, m, n, k, scale):
    """Operands, sums and draws in the same buffers, call after call: kernels that begin while those in front end read what these wrote."""
    times = 40
    xs = [values(m, k, 50 + i) for i in range(3)]
    b, sb = ctx.quantize_e4m3(values(n, k, 7) / 64, block_rows=128, scale=scale)
    u = torch.rand(m, 2, generator=torch.Generator().manual_seed(1)).to(DEV)

    def one(x):
        q, s = ctx.quantize_e4m3(x, scale=scale)
        d = ctx.matmul_e4m3(q, s, b, sb, out_dtype=torch.float32)
        torch.cuda.synchronize()
        return (d, *ctx.sample(d, u, temperature=50.0))
    want = [one(x) for x in xs]
    q, s = ctx.quantize_e4m3(xs[0], scale=scale)
    d = torch.empty(m, n, device=DEV)
    got = [(torch.empty_like(want[0][1]), torch.empty_like(want[0][2])) for _ in range(times)]

    def chain():
        for i, (idx, logp) in enumerate(got):
            ctx.quantize_e4m3(xs[i % 3], scale=scale, out=q, out_scale=s)
            ctx.matmul_e4m3(q, s, b, sb, out_dtype=torch.float32, out=d)
            ctx.sample(d, u, temperature=50.0, out_idx=idx, out_logp=logp)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for run in (chain, graph.replay, graph.replay):
        for idx, logp in got:
            idx.fill_(-7)
        run()
        for i, (idx, logp) in enumerate(got):
            assert torch.equal(idx, want[i % 3][1]) and torch.equal(logp, want[i % 3][2]), i
        assert torch.equal(d, want[(times - 1) % 3][0])


def quantised(x, block_rows, scale):
    q, s = lowbit.quantize(lowbit.as_float64(x), block_rows, scale)
    qt = torch.zeros(x.shape[0], -(-x.shape[1] // 16) * 16)
    qt[:, :x.shape[1]] = torch.from_numpy(q)
    dt = torch.float8_e8m0fnu if scale == "e8m0" else torch.float32
    return qt.to(torch.float8_e4m3fn).to(DEV)[:, :x.shape[1]], torch.from_numpy(s).float().to(dt).to(DEV), q, s


@pytest.mark.parametrize("signs", [False, True])
@pytest.mark.parametrize("scale", [torch.float32, torch.float8_e8m0fnu])
@pytest.mark.parametrize("m,n,k", [(40, 130, 1024), (1700, 515, 1024), (40, 130, 8192), (1700, 515, 4096), (1700, 260, 16384)])
def test_matmul_sums_that_24_bits_hold(ctx, m, n, k, scale, signs):
    """Values 1, 1.125, .. 1.875 with scales 1: products are multiples of 2^-6 below 4, a sum of 16,384 of them has 22 bits. Sums of
    24 bits are exact, in any order, rounded or cut; sums of fewer are not."""
    g = torch.Generator(device=DEV).manual_seed(k)

    def some(rows):
        v = 1 + torch.randint(0, 8, (rows, k), generator=g, device=DEV) / 8
        return v * (1 - 2 * torch.randint(0, 2, (rows, k), generator=g, device=DEV)) if signs else v
    a, b = some(m), some(n)
    sa, sb = torch.ones(m, k // 128, device=DEV).to(scale), torch.ones(-(-n // 128), k // 128, device=DEV).to(scale)
    got = ctx.matmul_e4m3(a.to(torch.float8_e4m3fn), sa, b.to(torch.float8_e4m3fn), sb, out_dtype=torch.float32)
    assert torch.equal(got.double(), a.double() @ b.double().t())


@pytest.mark.parametrize("positive", [False, True])
@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("m,n,k", [(40, 300, 1000), (1700, 515, 1000), (40, 300, 4296), (1700, 515, 4096), (1700, 515, 4296)])
def test_matmul_error_goes_with_the_additions(ctx, m, n, k, scale, positive):
    """An addition of the tensor core takes 32 of K: it cuts the sum below a unit of its 24 bits, and what it cuts off the 32 products
    is no more than another. The kernel with scales of two in its tiles adds k / 32 times (and a part of 4,096 of K to the next with one rounding);
    the others four times within a block, then a block with roundings of the scales' product and of the sum, and up to eight parts."""
    x, y = values(m, k, 31), values(n, k, 32)
    (a, sa, av, sav), (b, sb, bv, sbv) = (quantised(v.abs() if positive else v, r, scale) for v, r in ((x, 1), (y, 128)))
    want, mag = lowbit.matmul(av, sav, bv, sbv)
    got = lowbit.as_float64(ctx.matmul_e4m3(a, sa, b, sb, out_dtype=torch.float32))
    blocks = lowbit.blocks_of(k)
    in_tiles = scale == "e8m0" and (m > 1000 or (n <= 1024 and k <= 1024))
    units = 2 * -(-k // 32) + 1 if in_tiles else 8 + blocks / 2 + 2 + 4
    assert (np.abs(got - want) <= units * 2.0 ** -23 * mag).all(), (np.abs(got - want) / mag).max() * 2.0 ** 23
