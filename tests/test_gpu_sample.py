"""ks_sample against its definition in 64 bits."""
import numpy as np
import pytest
import torch

from tests import lowbit
from paper_2609_35587_b200 import binding as ks
from paper_2609_35587_b200 import workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda"
SETTINGS = [dict(), dict(t=0.7), dict(top_k=5), dict(top_k=1), dict(top_p=0.8), dict(top_p=0.01), dict(min_p=0.1), dict(min_p=1.0),
            dict(t=1.3, top_k=40, top_p=0.9), dict(t=0.5, top_k=100, top_p=0.95, min_p=0.02), dict(t=0.0), dict(t=0.01),
            dict(t=50.0, top_p=0.5), dict(top_k=10 ** 9)]


@pytest.fixture(scope="module")
def ctx():
    c = ks.Context(wl.gpu_desc(), 0)
    yield c
    assert c.device_status() == ks.KS_OK
    c.close()


def draw(ctx, scores, u, seg_off=None, params=None, **s):
    kw = {{"t": "temperature"}.get(k, k): v for k, v in s.items()}
    return ctx.sample(scores, u, d_seg_off=seg_off, params=params, **kw)


def numbers(p, draws, seed):
    u = torch.rand(p, draws, generator=torch.Generator().manual_seed(seed))
    u.view(-1)[0] = 0.0
    u.view(-1)[-1] = 1 - 2.0 ** -24
    return u.to(DEV)


def check(scores, u, idx, logp, rows=None, settings=None, **s):
    x, un, i, lp = lowbit.as_float64(scores), u.cpu().numpy(), idx.cpu().numpy(), logp.cpu().numpy()
    for r in range(len(un)):
        row = x[r] if rows is None else x[rows[r]:rows[r + 1]]
        lowbit.check_draws(row, un[r], i[r], lp[r], **(s if settings is None else settings[r]))


@pytest.mark.parametrize("s", SETTINGS, ids=str)
@pytest.mark.parametrize("p,c,spread", [(3, 1, 1.0), (4, 7, 2.0), (2, 31, 0.0), (5, 1000, 3.0), (2, 5000, 0.05), (2, 2049, 10.0)])
def test_settings(ctx, p, c, spread, s):
    g = torch.Generator().manual_seed(c)
    x = (torch.randn(p, c, generator=g) * spread).to(DEV)
    u = numbers(p, 7, c)
    idx, logp = draw(ctx, x, u, **s)
    check(x, u, idx, logp, **s)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("c", [257, 4096, 33333, 131072])
@pytest.mark.parametrize("s", [dict(t=0.8, top_p=0.9), dict(top_k=50), dict(t=1.5, top_k=1000, top_p=0.7, min_p=0.01)], ids=str)
def test_types_and_lengths(ctx, c, dtype, s):
    """16-bit scores have many ties; rows of odd length begin at odd addresses."""
    g = torch.Generator().manual_seed(c + 1)
    x = (torch.randn(3, c, generator=g) * 2.5).to(dtype).to(DEV)
    u = numbers(3, 8, c)
    idx, logp = draw(ctx, x, u, **s)
    check(x, u, idx, logp, **s)


@pytest.mark.parametrize("c", [534600, 1200007])
def test_long_rows(ctx, c):
    """The whole search space, and more than any on-chip memory holds."""
    g = torch.Generator().manual_seed(c)
    x = (torch.randn(1, c, generator=g) * 2).to(DEV)
    u = numbers(1, 5, c)
    for s in (dict(), dict(t=0.9, top_k=3000, top_p=0.9)):
        idx, logp = draw(ctx, x, u, **s)
        check(x, u, idx, logp, **s)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("s", SETTINGS, ids=str)
def test_masked_rows(ctx, dtype, s):
    """Rows without a candidate, with one, with the type's lowest value as a mask, with infinities and numbers that are none."""
    c = 300
    low = torch.finfo(dtype).min
    x = (torch.randn(9, c, generator=torch.Generator().manual_seed(2)) * 2).to(dtype)
    x[0] = -np.inf
    x[1] = np.nan
    x[2, :] = -np.inf
    x[2, 17] = -3.0
    x[3, 5:] = low
    x[4] = low
    x[5, 7:200] = np.nan
    x[6, 11], x[6, 290] = np.inf, np.inf
    x[7, ::2] = -np.inf
    x[8] = 0.0
    x[8, 100:] = -0.0
    x, u = x.to(DEV), numbers(9, 6, 1)
    idx, logp = draw(ctx, x, u, **s)
    check(x, u, idx, logp, **s)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_segments_with_settings_of_their_own(ctx, dtype):
    """Empty and ragged segments; settings out of range in device memory count as the header says."""
    lens = [0, 1, 5, 0, 700, 33, 2048, 4097, 1, 0, 9000, 3, 0]
    rows = np.concatenate([[0], np.cumsum(lens)])
    x = (torch.randn(int(rows[-1]), generator=torch.Generator().manual_seed(3)) * 2).to(dtype).to(DEV)
    rng = np.random.RandomState(1)
    rec = np.zeros(len(lens), ks.SAMPLING_DT)
    rec["temperature"] = rng.uniform(0.3, 2.0, len(lens))
    rec["top_k"] = rng.randint(0, 60, len(lens))
    rec["top_p"] = rng.uniform(0.3, 1.0, len(lens))
    rec["min_p"] = rng.uniform(0.0, 0.1, len(lens))
    rec[4] = (-1.0, 3, 0.5, 0.0)       # as temperature 0
    rec[6] = (np.nan, 3, 0.5, 0.0)     # the same
    rec[5] = (1.0, -7, 2.0, -1.0)      # everything stays
    rec[7] = (1.0, 0, -0.5, np.nan)    # the best alone; min_p of no number as 0
    rec[10] = (0.8, 0, np.nan, 3.0)    # no top-p; min_p as 1
    u = numbers(len(lens), 3, 5)
    off = torch.from_numpy(rows).to(DEV)
    idx, logp = draw(ctx, x, u, seg_off=off, params=ks.to_device(rec, DEV))
    settings = [dict(t=r["temperature"], top_k=int(r["top_k"]), top_p=r["top_p"], min_p=r["min_p"]) for r in rec]
    settings[4] = settings[6] = dict(t=0.0)
    settings[5] = dict(t=1.0)
    settings[7] = dict(t=1.0, top_k=1)
    settings[10] = dict(t=rec[10]["temperature"], min_p=1.0)
    check(x, u, idx, logp, rows=rows, settings=settings)


def test_strided_rows_and_guards(ctx):
    big = torch.randn(20, 999, generator=torch.Generator().manual_seed(4)).to(DEV)
    x = big[3:17, 5:700]
    u = numbers(14, 4, 2)
    out = torch.full((16, 4), 77, dtype=torch.int32, device=DEV)
    lp = torch.full((16, 4), 77.0, device=DEV)
    idx, logp = ctx.sample(x, u, top_p=0.9, out_idx=out[:14], out_logp=lp[:14])
    check(x, u, idx, logp, top_p=0.9)
    assert bool((out[14:] == 77).all()) and bool((lp[14:] == 77).all())
    again, none = ctx.sample(x, u, top_p=0.9, out_idx=torch.empty_like(idx), out_logp=None)
    assert none is None and torch.equal(again, idx)


def test_random_numbers_out_of_range(ctx):
    x = torch.randn(2, 50, generator=torch.Generator().manual_seed(6)).to(DEV)
    u = torch.tensor([[-1.0, 1.0, 5.0], [float("nan"), 0.0, float("inf")]], device=DEV)
    idx, _ = ctx.sample(x, u)
    assert idx.tolist() == [[0, 49, 49], [0, 0, 49]]


def test_many_rows(ctx):
    """More rows than the machine holds at once, all lengths of draws."""
    x = (torch.randn(3000, 70, generator=torch.Generator().manual_seed(8)) * 2).to(DEV)
    u = numbers(3000, ks.KS_MAX_K, 9)
    idx, logp = draw(ctx, x, u, t=0.9, top_k=20, top_p=0.9)
    check(x, u, idx, logp, t=0.9, top_k=20, top_p=0.9)


def test_frequencies(ctx):
    """Over a grid of numbers a candidate is drawn as often as its probability says."""
    x = torch.randn(1, 40, generator=torch.Generator().manual_seed(10)).to(DEV)
    n = 1 << 14
    u = ((torch.arange(n) + 0.5) / n).view(-1, 32).to(DEV)
    idx, _ = ctx.sample(x.expand(n // 32, 40).contiguous(), u, temperature=0.8)
    got = np.bincount(idx.cpu().numpy().ravel(), minlength=40)
    w = lowbit.distribution(lowbit.as_float64(x)[0], t=0.8)
    assert np.abs(got - n * w / w.sum()).max() <= 1.0 + 1e-6  # a stretch of the grid holds its length in points, to one


def test_same_bits_in_streams_and_graphs(ctx):
    x = torch.randn(5, 20000, generator=torch.Generator().manual_seed(11)).to(DEV)
    u = numbers(5, 4, 12)
    first = ctx.sample(x, u, top_k=200, top_p=0.9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = ctx.sample(x, u, top_k=200, top_p=0.9)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first[0], second[0]) and torch.equal(first[1], second[1])
    idx, lp = torch.empty_like(first[0]), torch.empty_like(first[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.sample(x, u, top_k=200, top_p=0.9, out_idx=idx, out_logp=lp)
    for seed in (1, 2):
        x.copy_(torch.randn(5, 20000, generator=torch.Generator().manual_seed(seed)).to(DEV))
        u.copy_(numbers(5, 4, seed))
        graph.replay()
        check(x, u, idx, lp, top_k=200, top_p=0.9)


def test_one_pass_quantised_layer_scored_and_drawn(ctx):
    """Rows through two layers in eight bits, and candidates drawn from what comes out."""
    g = torch.Generator().manual_seed(13)
    rows, wide, per = 600, 256, 200
    x = torch.randn(rows, 64, generator=g).to(DEV)
    w1, w2 = torch.randn(wide, 64, generator=g).to(DEV) / 8, torch.randn(1, wide, generator=g).to(DEV) / 16
    q, s = ctx.quantize_e4m3(x)
    q1, s1 = ctx.quantize_e4m3(w1, block_rows=128)
    q2, s2 = ctx.quantize_e4m3(w2, block_rows=128)
    h, hs = ctx.matmul_e4m3(q, s, q1, s1, relu=True, out_dtype=torch.float8_e4m3fn)
    scores = ctx.matmul_e4m3(h, hs, q2, s2, out_dtype=torch.float32)
    want, mag = lowbit.matmul(lowbit.as_float64(h), lowbit.as_float64(hs), lowbit.as_float64(q2), lowbit.as_float64(s2))
    assert (np.abs(lowbit.as_float64(scores) - want) <= (wide + 6) * 2.0 ** -23 * mag + 2.0 ** -24 * np.abs(want)).all()
    off = torch.arange(0, rows + 1, per, dtype=torch.int64, device=DEV)
    u = numbers(rows // per, 8, 14)
    idx, logp = ctx.sample(scores.view(-1), u, temperature=0.3, top_k=20, d_seg_off=off)
    check(scores.view(-1), u, idx, logp, rows=off.cpu().numpy(), t=0.3, top_k=20)


def test_rows_without_a_score(ctx):
    """No columns, segments that are all empty, no rows."""
    u = numbers(3, 2, 1)
    idx, logp = ctx.sample(torch.empty(3, 0, device=DEV), u, top_p=0.5)
    assert idx.tolist() == [[-1, -1]] * 3 and bool((logp == -np.inf).all())
    idx, logp = ctx.sample(torch.empty(0, device=DEV), u, top_k=4, d_seg_off=torch.zeros(4, dtype=torch.int64, device=DEV))
    assert idx.tolist() == [[-1, -1]] * 3 and bool((logp == -np.inf).all())
    idx, _ = ctx.sample(torch.empty(0, 5, device=DEV), torch.empty(0, 2, device=DEV))
    assert idx.shape == (0, 2)


@pytest.mark.parametrize("p,c", [(1, 3000), (2, 60000), (300, 3000), (300, 20000), (1, 1000003)])
@pytest.mark.parametrize("s", [dict(top_p=0.6), dict(top_k=700, top_p=0.8), dict(top_k=300), dict(top_k=2000, min_p=0.01)], ids=str)
@pytest.mark.parametrize("values", ["equal", "two", "steps", "far", "huge"])
def test_scores_that_crowd(ctx, p, c, s, values):
    """Scores of which far more than a sorted list holds share a bin or a value, or lie where fp32 has no more room."""
    g = torch.Generator().manual_seed(c)
    x = {"equal": torch.full((p, c), 1.5), "two": torch.randint(0, 2, (p, c), generator=g).float(),
         "steps": torch.randint(0, 7, (p, c), generator=g).float() * 0.25,
         "far": torch.where(torch.rand(p, c, generator=g) < 0.001, torch.tensor(0.0), torch.tensor(-30.0)),
         "huge": torch.randn(p, c, generator=g) * 1e37}[values]
    x = x.to(DEV)
    u = numbers(p, 3, p)
    idx, logp = draw(ctx, x, u, **s)
    rows = range(p) if p < 10 else range(0, p, 60)
    for r in rows:
        lowbit.check_draws(lowbit.as_float64(x[r]), u[r].cpu().numpy(), idx[r].cpu().numpy(), logp[r].cpu().numpy(), **s)


@pytest.mark.parametrize("t", [1e-38, 1e-3, 1e30, float("inf")])
def test_temperatures_from_device_memory(ctx, t):
    """Very small ones leave the best score, very large ones make all alike; settings of device memory are not refused."""
    x = torch.randn(3, 500, generator=torch.Generator().manual_seed(3))
    x[1, 7] = x[1, 400] = 9.0
    x[2, 3] = -np.inf
    x = x.to(DEV)
    rec = np.zeros(3, ks.SAMPLING_DT)
    rec["temperature"], rec["top_p"] = t, 0.9
    u = numbers(3, 4, 2)
    idx, logp = ctx.sample(x, u, params=ks.to_device(rec, DEV))
    check(x, u, idx, logp, t=t, top_p=0.9)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("c", [1, 2, 32, 33, 63, 64, 65, 128, 129, 255, 256, 257, 300])
@pytest.mark.parametrize("s", [dict(), dict(top_p=0.7, min_p=0.05), dict(top_k=33, top_p=0.9), dict(t=0.0), dict(min_p=1.0)], ids=str)
def test_short_rows(ctx, c, dtype, s):
    """The same draws from few rows, from many, and from segments among longer ones."""
    g = torch.Generator().manual_seed(c)
    p, few = 330, 5
    x = (torch.randn(p, c, generator=g) * 2).to(dtype)
    x[1, c // 2], x[2, 0], x[3, c - 1] = float("nan"), float("inf"), -float("inf")
    x[4] = -float("inf")
    x[0] = x[0, 0]
    x = x.to(DEV)
    u = numbers(p, 33 if c == 64 else 3, c)[:, :32].contiguous()
    idx, logp = draw(ctx, x, u, **s)
    check(x[:few], u[:few], idx[:few], logp[:few], **s)
    check(x[-few:], u[-few:], idx[-few:], logp[-few:], **s)
    again = draw(ctx, x[:few].contiguous(), u[:few].contiguous(), **s)
    assert torch.equal(again[0], idx[:few]) and torch.equal(again[1], logp[:few])
    long = torch.randn(3000, generator=g).to(dtype).to(DEV)
    flat = torch.cat([torch.cat([x[r], long]) for r in range(few)])
    lens = torch.tensor([0] + [c, 3000] * few, dtype=torch.int64)
    seg = draw(ctx, flat, u[:few].repeat_interleave(2, 0).contiguous(), seg_off=lens.cumsum(0).to(DEV), **s)
    assert torch.equal(seg[0][::2], idx[:few]) and torch.equal(seg[1][::2], logp[:few])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("p,c", [(1, 400000), (20, 200000), (300, 130000)])
@pytest.mark.parametrize("s", [dict(top_p=0.9), dict(top_p=0.3, t=0.8, min_p=0.001), dict(top_k=100000, top_p=0.8), dict(top_p=0.999, t=2.0)], ids=str)
@pytest.mark.parametrize("spread", [0.05, 1.0, 3.0])
def test_many_scores_around_the_cut(ctx, p, c, dtype, s, spread):
    """Long rows in which a bin of the histogram around top-p's cut holds more candidates than are listed."""
    x = (torch.randn(p, c, generator=torch.Generator(device=DEV).manual_seed(c), device=DEV) * spread).to(dtype)
    u = numbers(p, 4, 3)
    idx, logp = draw(ctx, x, u, **s)
    for r in ([0] if p == 1 else [0, p - 1]):
        lowbit.check_draws(lowbit.as_float64(x[r]), u[r].cpu().numpy(), idx[r].cpu().numpy(), logp[r].cpu().numpy(), **s)


def raw(ctx, scores, c, off, u, idx, logp, **s):
    """The C call with a total of its own."""
    one = ks._Sampling(s.get("t", 1.0), s.get("top_k", 0), s.get("top_p", 1.0), s.get("min_p", 0.0))
    st = ks._lib.ks_sample(ctx._h, scores.data_ptr(), ks._TYPES[scores.dtype], u.shape[0], c, 0, off.data_ptr(), ks.ctypes.byref(one), None,
                           u.data_ptr(), u.shape[1], idx.data_ptr(), logp.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert st == ks.KS_OK


@pytest.mark.parametrize("c", [0, 1, 200, 256, 257, 10 ** 6])
@pytest.mark.parametrize("s", [dict(), dict(top_k=9), dict(top_p=0.8, min_p=0.01)], ids=str)
def test_total_of_segments_decides_no_draw(ctx, c, s):
    """Rows are as long as the offsets say, whatever the call was told about their total; also where a replayed graph finds others."""
    lens = [[3, 256, 0, 5, 90], [900, 0, 257, 5, 4000], [0, 0, 256, 60000, 1]]
    x = (torch.randn(61000, generator=torch.Generator().manual_seed(21)) * 2).to(DEV)
    offs = [torch.tensor([0] + n, dtype=torch.int64).cumsum(0).to(DEV) for n in lens]
    u = numbers(5, 6, 4)
    off = offs[0].clone()
    idx, lp = torch.full((5, 6), 77, dtype=torch.int32, device=DEV), torch.full((5, 6), 77.0, device=DEV)
    raw(ctx, x, c, off, u, idx, lp, **s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        raw(ctx, x, c, off, u, idx, lp, **s)
    for o in offs:
        off.copy_(o)
        idx.fill_(77)
        lp.fill_(77.0)
        graph.replay()
        check(x, u, idx, lp, rows=o.cpu().numpy(), **s)
        want = ctx.sample(x, u, d_seg_off=o, **{{"t": "temperature"}.get(k, k): v for k, v in s.items()})
        assert torch.equal(idx, want[0]) and torch.equal(lp, want[1])


def test_segments_without_scores(ctx):
    """No scores at all (a tensor without elements has no address), though the offsets name some: nothing is read."""
    none = torch.empty(0, device=DEV)
    assert none.data_ptr() == 0
    off = torch.tensor([0, 300, 300, 700], dtype=torch.int64, device=DEV)
    idx, logp = ctx.sample(none, numbers(3, 2, 1), d_seg_off=off)
    assert idx.tolist() == [[-1, -1]] * 3 and bool((logp == -np.inf).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("mean", ["short", "long"])
@pytest.mark.parametrize("s", [None, dict(t=0.8, top_p=0.9), dict(top_k=60), dict()], ids=str)
def test_many_segments(ctx, dtype, mean, s):
    """As many segments as a CTA each takes: short ones of a launch of their own, ones that are kept on chip, ones that are not, and (long on
    the average) none that are; settings of the call or of each row."""
    p = 400
    rng = np.random.RandomState(5)
    lens = np.exp(rng.uniform(0, np.log(1500), p)).astype(np.int64)
    lens[rng.rand(p) < 0.05] = 0
    lens[:12] = [255, 256, 257, 258, 511, 512, 513, 1024, 1025, 7169, 14337, 30000]
    if mean == "long":
        lens[20:80] = rng.randint(60000, 140000, 60)
    rng.shuffle(lens)
    rows = np.concatenate([[0], np.cumsum(lens)])
    x = (torch.randn(int(rows[-1]), generator=torch.Generator().manual_seed(31)) * 2).to(dtype)
    x[torch.rand(len(x), generator=torch.Generator().manual_seed(32)) < 0.05] = -float("inf")
    x, u, off = x.to(DEV), numbers(p, 5, 33), torch.from_numpy(rows).to(DEV)
    if s is None:
        rec = np.zeros(p, ks.SAMPLING_DT)
        rec["temperature"], rec["top_k"] = rng.uniform(0.3, 2.0, p), rng.randint(0, 200, p)
        rec["top_p"], rec["min_p"] = rng.uniform(0.3, 1.1, p), rng.uniform(-0.05, 0.05, p)
        rec["temperature"][rng.rand(p) < 0.1] = 0.0
        idx, logp = draw(ctx, x, u, seg_off=off, params=ks.to_device(rec, DEV))
        settings = [dict(t=r["temperature"], top_k=int(r["top_k"]), top_p=min(r["top_p"], 1.0), min_p=max(r["min_p"], 0.0)) for r in rec]
    else:
        idx, logp = draw(ctx, x, u, seg_off=off, **s)
        settings = [s] * p
    xs, un, i, lp = lowbit.as_float64(x), u.cpu().numpy(), idx.cpu().numpy(), logp.cpu().numpy()
    for r in range(p):
        if lens[r] < 20000 or r % 8 == 0:
            lowbit.check_draws(xs[rows[r]:rows[r + 1]], un[r], i[r], lp[r], **settings[r])
