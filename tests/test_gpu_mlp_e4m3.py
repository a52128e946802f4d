"""Rankers held in eight bits (ks_model_create_mlp_e4m3): their scores are those of their layers taken one by one through
ks_quantize_e4m3 and ks_matmul_e4m3, which tests of their own hold to the definition; the first layer's input and the last layer
are held to it here."""
import numpy as np
import pytest
import torch

from tests import lowbit
from paper_2609_35587_b200 import binding as ks
from paper_2609_35587_b200 import workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda"
DESC = wl.gpu_desc()
BATCH = 2 * 74 * 256  # rows that the layers take at a time


@pytest.fixture(scope="module")
def ctx():
    c = ks.Context(DESC, 0)
    yield c
    assert c.device_status() == ks.KS_OK
    c.close()


def make(onehot, hidden, seed):
    st = wl.feature_stats("cfg2")
    mu, sg = wl.onehot_stats(st["mu"], st["sigma"]) if onehot else (st["mu"], st["sigma"])
    return wl.mlp_xavier(seed, [80 if onehot else 64] + hidden + [1], mu, sg)


def features(ctx, P, C, seed=4):
    w = wl.make_workload(2, P=P, C=C, trees=4, depth=2)
    d_p, d_c = ks.to_device(w.problems, torch.device(DEV)), ks.to_device(w.candidates, torch.device(DEV))
    return w, d_p, d_c, ctx.featurize(d_p, P, d_c, C)


def expanded(x, onehot):
    """The model's input positions, as numpy fp32."""
    x = x.cpu().numpy()
    if not onehot:
        return np.concatenate([x[:, :63], np.zeros((len(x), 1), np.float32)], 1)
    keep = [c for c in range(63) if c not in (5, 9, 17, 18)]
    ind = [(x[:, [c]] == np.arange(n)).astype(np.float32) for c, n in ((5, 4), (9, 3), (17, 4), (18, 3))]
    return np.concatenate([x[:, keep]] + ind + [np.zeros((len(x), 7), np.float32)], 1).astype(np.float32)


def standardised(x, mlp, onehot):
    v = expanded(x, onehot)
    v = np.where(np.isfinite(v), v, np.float32(0))
    v = (v - np.asarray(mlp["mu"], np.float32)) / np.asarray(mlp["sigma"], np.float32)
    used = 73 if onehot else 63
    v[:, used:] = 0
    return torch.from_numpy(np.ascontiguousarray(v, np.float32)).to(DEV)


def by_layers(ctx, x, mlp, onehot):
    """(scores in 64 bits from the last hidden layer, what fp32 sums of them may be off by)."""
    a, sa = ctx.quantize_e4m3(standardised(x, mlp, onehot))
    want_q, want_s = lowbit.quantize(lowbit.as_float64(standardised(x, mlp, onehot)), 1, "e8m0")
    np.testing.assert_array_equal(lowbit.as_float64(a), want_q)
    np.testing.assert_array_equal(lowbit.as_float64(sa), want_s)
    widths = mlp["widths"]
    for l in range(len(widths) - 2):
        w = torch.from_numpy(np.asarray(mlp["weights"][l], np.uint16).reshape(widths[l + 1], widths[l]).view(np.int16)).view(torch.bfloat16).to(DEV)
        b, sb = ctx.quantize_e4m3(w, block_rows=128)
        bias = torch.from_numpy(np.asarray(mlp["biases"][l], np.float32)).to(DEV)
        if l + 3 < len(widths):
            a, sa = ctx.matmul_e4m3(a, sa, b, sb, bias=bias, relu=True, out_dtype=torch.float8_e4m3fn)
        else:
            h = ctx.matmul_e4m3(a, sa, b, sb, bias=bias, relu=True, out_dtype=torch.bfloat16)
    h = lowbit.as_float64(h)
    w = lowbit.as_float64(torch.from_numpy(np.asarray(mlp["weights"][-1], np.uint16).reshape(-1).view(np.int16)).view(torch.bfloat16))
    b = float(np.float32(mlp["biases"][-1][0]))
    return h @ w + b, (len(w) + 2) * 2.0 ** -24 * (np.abs(h) @ np.abs(w) + abs(b))


@pytest.mark.parametrize("onehot", [False, True])
@pytest.mark.parametrize("hidden", [[64], [128], [256, 256], [192, 320], [1024, 1024, 512, 256], [64, 128, 192, 256, 64]])
@pytest.mark.parametrize("P,C", [(1, 1), (1, 60), (2, 70), (3, 300)])
def test_scores(ctx, onehot, hidden, P, C):
    mlp = make(onehot, hidden, len(hidden))
    model = ctx.model_create_mlp_e4m3(mlp)
    assert "matmul_scaled_kernel" in model.describe()
    _, _, _, x = features(ctx, P, C)
    x[0, 40], x[0, 41] = float("nan"), float("inf")
    got = lowbit.as_float64(ctx.score(x, model))
    want, tol = by_layers(ctx, x, mlp, onehot)
    assert (np.abs(got - want) <= tol).all()


def test_scores_of_several_batches(ctx):
    mlp = make(False, [256, 128], 3)
    model = ctx.model_create_mlp_e4m3(mlp)
    _, _, _, x = features(ctx, 10, 4000)
    got = lowbit.as_float64(ctx.score(x, model))
    parts = [by_layers(ctx, x[i:i + BATCH], mlp, False) for i in range(0, len(x), BATCH)]
    want, tol = (np.concatenate([p[j] for p in parts]) for j in (0, 1))
    assert len(parts) == 2 and (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("onehot", [False, True])
def test_select_ranks_the_same_scores(ctx, onehot):
    P, C, k = 3, 700, 10
    model = ctx.model_create_mlp_e4m3(make(onehot, [256, 128], 5))
    w, d_p, d_c, x = features(ctx, P, C)
    scores = ctx.score(x, model).cpu().numpy().reshape(P, C)
    idx, sc = (t.cpu().numpy() for t in ctx.select(d_p, P, d_c, C, model, k))
    for i in range(P):
        order = np.lexsort((np.arange(C), -scores[i]))[:k]
        np.testing.assert_array_equal(idx[i], order)
        np.testing.assert_array_equal(sc[i], scores[i][order])
    # the other calls of the path
    h_idx, h_sc = ctx.select_host(w.problems, P, w.candidates, C, model, k)
    np.testing.assert_array_equal(h_idx.numpy(), idx)
    np.testing.assert_array_equal(h_sc.numpy(), sc)
    one_i, one_s = ctx.select_one(w.problems[1:2], d_c, C, model, k)
    lone = ctx.score(x[C:2 * C].contiguous(), model).cpu().numpy()
    order = np.lexsort((np.arange(C), -lone))[:k]
    np.testing.assert_array_equal(one_i.numpy(), order)
    np.testing.assert_array_equal(one_s.numpy(), lone[order])


def test_select_by_segments_then_draw(ctx):
    """Candidate sets of their own, ranked and drawn from: the draws of temperature 0 are the best candidates."""
    P, C = 5, 400
    model = ctx.model_create_mlp_e4m3(make(False, [128, 64], 6))
    w = wl.make_workload(2, P=P, C=C, trees=4, depth=2)
    d_p, d_c = ks.to_device(w.problems, torch.device(DEV)), ks.to_device(w.candidates, torch.device(DEV))
    lens = [130, 0, 400, 7, 1]
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)).to(DEV)
    idx = torch.cat([torch.randperm(C, generator=torch.Generator().manual_seed(i))[:n] for i, n in enumerate(lens)]).int().to(DEV)
    pairs = int(off[-1])
    x = ctx.featurize(d_p, P, d_c, C, off, idx, pairs)
    scores = ctx.score(x, model)
    top, _ = ctx.select(d_p, P, d_c, C, model, 1, off, idx, pairs)
    u = torch.rand(P, 4, generator=torch.Generator().manual_seed(1)).to(DEV)
    at, _ = ctx.sample(scores, u, temperature=0.0, d_seg_off=off)
    for i, n in enumerate(lens):
        if n == 0:
            assert at[i].tolist() == [-1] * 4 and int(top[i, 0]) == -1
            continue
        s = scores[int(off[i]):int(off[i + 1])]
        best = s == s.max()
        # (ks_select goes by pool index among equal scores, a draw by place in the segment)
        assert int(top[i, 0]) == int(idx[int(off[i]):int(off[i + 1])][best].min())
        assert set(at[i].tolist()) == {int(torch.nonzero(best)[0, 0])}
    at, logp = ctx.sample(scores, u, temperature=0.5, top_k=20, top_p=0.9, d_seg_off=off)
    rows = off.cpu().numpy()
    for i in range(P):
        lowbit.check_draws(lowbit.as_float64(scores)[rows[i]:rows[i + 1]], u.cpu().numpy()[i], at.cpu().numpy()[i],
                           logp.cpu().numpy()[i], t=0.5, top_k=20, top_p=0.9)


def test_little_workspace(ctx):
    """Where the memory for whole batches cannot be had, fewer rows at a time, with scores that agree to the layers' sums."""
    model = ctx.model_create_mlp_e4m3(make(False, [1024, 512], 7))
    _, _, _, x = features(ctx, 2, 3000)
    want = ctx.score(x, model)
    small = ks.Context(DESC, 0)
    model2 = small.model_create_mlp_e4m3(make(False, [1024, 512], 7))
    small.debug_limit_workspace(8 << 20)
    got = small.score(x, model2)
    assert small.device_status() == ks.KS_OK
    assert torch.equal(got, want)


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("m", [5, 300, 4200])
def test_wait_that_runs_out(m, scale):
    """Copies that never come: the kernel gives up in bounded time, the call's status says so, and the next call is right."""
    c = ks.Context(DESC, 0)
    g = torch.Generator().manual_seed(2)
    a, b = torch.randn(m, 300, generator=g).to(DEV), torch.randn(200, 300, generator=g).to(DEV)
    qa, qb = c.quantize_e4m3(a, scale=scale), c.quantize_e4m3(b, block_rows=128, scale=scale)
    want = c.matmul_e4m3(*qa, *qb)
    c.debug_set_wait(50, 1)
    c.matmul_e4m3(*qa, *qb)
    assert c.device_status() == ks.KS_ERR_TIMEOUT
    c.debug_set_wait(0, 0)
    assert torch.equal(c.matmul_e4m3(*qa, *qb), want)
    assert c.device_status() == ks.KS_OK
    c.close()


@pytest.mark.parametrize("onehot,hidden", [(False, [128]), (True, [64]), (False, [256, 128]), (False, [192, 320]), (True, [1024, 1024, 512, 256])])
def test_a_row_scores_the_same_whatever_is_beside_it(ctx, onehot, hidden):
    """Alone, among a few, in a full batch, in the rest behind one, and with little workspace: equal bits."""
    mlp = make(onehot, hidden, 9)
    model = ctx.model_create_mlp_e4m3(mlp)
    _, _, _, x = features(ctx, 4, 5000)
    base = ctx.score(x, model)
    for rows in (1, 16, 17, 65, 500, 4000):
        for first in range(0, len(x), 2500):
            part = x[first:first + rows].contiguous()
            assert torch.equal(ctx.score(part, model), base[first:first + len(part)]), (rows, first)
    at = torch.arange(BATCH + 2112, device=DEV) % len(x)
    assert torch.equal(ctx.score(x[at], model), base[at])
    small = ks.Context(DESC, 0)
    model2 = small.model_create_mlp_e4m3(mlp)
    small.debug_limit_workspace(8 << 20)
    assert torch.equal(small.score(x[at], model2), base[at])
    assert small.device_status() == ks.KS_OK
    small.close()


@pytest.mark.parametrize("hidden", [[128], [256, 128], [1024, 512]])
def test_select_over_several_batches(ctx, hidden):
    """Copies of the best candidates lie in the rest behind the first batch: they score the same, and the lower index comes first."""
    k, rest = 32, 2112
    model = ctx.model_create_mlp_e4m3(make(False, hidden, 10))
    w = wl.make_workload(2, P=1, C=BATCH, trees=4, depth=2)
    d_p, d_c = ks.to_device(w.problems, torch.device(DEV)), ks.to_device(w.candidates, torch.device(DEV))
    first = ctx.score(ctx.featurize(d_p, 1, d_c, BATCH), model).cpu().numpy()
    order = np.lexsort((np.arange(BATCH), -first))
    pool = np.concatenate([w.candidates, w.candidates[order[:rest]]])
    d_c = ks.to_device(pool, torch.device(DEV))
    scores = ctx.score(ctx.featurize(d_p, 1, d_c, len(pool)), model).cpu().numpy()
    np.testing.assert_array_equal(scores, np.concatenate([first, first[order[:rest]]]))
    want = np.lexsort((np.arange(len(pool)), -scores))[:k]
    for idx, sc in ((t.cpu().numpy() for t in ctx.select(d_p, 1, d_c, len(pool), model, k)),
                    (t.cpu().numpy()[None] for t in ctx.select_one(w.problems[:1], d_c, len(pool), model, k))):
        np.testing.assert_array_equal(idx[0], want)
        np.testing.assert_array_equal(sc[0], scores[want])
    few = order[:40]  # the same candidates as a small pool
    idx, sc = (t.cpu().numpy() for t in ctx.select_one(w.problems[:1], ks.to_device(w.candidates[few], torch.device(DEV)), len(few), model, 8))
    np.testing.assert_array_equal(sc, first[few][:8])
    assert (first[few[idx]] == sc).all()
