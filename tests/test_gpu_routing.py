"""Routing to experts on the GPU: choice, weights, expert order and gradient, against plain forms in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2512_02551_b200 import hgemm, routing  # noqa: E402

TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "these tests need a B200"
    with hgemm.Context(0) as c:
        yield c


def scores64(l, score):
    if score == "sigmoid":
        return 1.0 / (1.0 + np.exp(-l))
    m = l.max(-1, keepdims=True)
    e = np.exp(l - np.where(np.isfinite(m), m, 0.0))
    return e / np.maximum(e.sum(-1, keepdims=True), 1e-300)


def values64(l, r):
    """What the choice goes by, -infinity for experts of groups that are left out (which groups: from the GPU's own choice where
    two groups are within rounding of one another is not needed: inputs keep them apart)."""
    s = scores64(l, r["score"])
    v = s + r["bias"] if r["bias"] is not None else (l if r["score"] == "softmax" else s)
    v = np.where(np.isnan(v), -np.inf, v)
    if r["groups"] > 1:
        T, E = v.shape
        g = v.reshape(T, r["groups"], -1)
        top = np.sort(g, -1)[..., ::-1]
        of = top[..., 0] + top[..., 1] if r["group_score"] == "top2" else top[..., 0]
        order = np.argsort(-of, -1, kind="stable")[:, :r["top_groups"]]
        keep = np.zeros(of.shape, dtype=bool)
        np.put_along_axis(keep, order, True, -1)
        v = np.where(keep[..., None], g, -np.inf).reshape(T, E)
    return s, v


RULES = [
    # experts, top_k, score, bias, groups, top_groups, group_score, renormalize, scale
    (1, 1, "softmax", False, 1, 1, "max", True, 1.0),
    (8, 2, "softmax", False, 1, 1, "max", True, 1.0),
    (8, 8, "sigmoid", False, 1, 1, "max", False, 0.5),
    (60, 4, "softmax", False, 4, 2, "max", False, 1.0),
    (64, 6, "softmax", True, 1, 1, "max", True, 1.0),
    (33, 32, "sigmoid", True, 1, 1, "max", True, 1.0),
    (128, 8, "softmax", False, 8, 3, "max", False, 16.0),
    (160, 6, "sigmoid", True, 8, 3, "max", True, 1.0),
    (256, 8, "sigmoid", True, 8, 4, "top2", True, 2.5),
    (512, 10, "sigmoid", False, 32, 4, "top2", True, 1.0),
    (511, 7, "softmax", False, 7, 1, "max", True, 1.0),
]


def rule(t):
    return dict(zip(("experts", "top_k", "score", "bias", "groups", "top_groups", "group_score", "renormalize", "scale"), t))


def make(ctx, r):
    return routing.Router(ctx, r["experts"], r["top_k"], score=r["score"], groups=r["groups"], top_groups=r["top_groups"], group_score=r["group_score"],
                          renormalize=r["renormalize"], scale=r["scale"])


def run(router, logits, bias=None):
    T = logits.shape[0]
    w = torch.full((T, router.top_k), float("nan"), device="cuda")
    i = torch.full((T, router.top_k), -7, dtype=torch.int32, device="cuda")
    router.forward(logits, w, i, bias=bias)
    return w, i


@pytest.mark.parametrize("t", RULES, ids=str)
@pytest.mark.parametrize("T", [1, 3, 130])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_choice_and_weights(ctx, t, T, dtype):
    """Every choice is among the largest eligible values up to rounding (2^-22: a score's exponential, division and the bias's
    addition, each within a few 2^-24), best first; the weights are those of the chosen experts."""
    r = rule(t)
    g = torch.Generator(device="cuda").manual_seed(T * 1000 + r["experts"])
    E, k = r["experts"], r["top_k"]
    logits = torch.randn(T, E + 3, generator=g, device="cuda").mul(2.0).to(dtype)[:, :E]     # rows further apart than they are wide
    bias = torch.randn(E, generator=g, device="cuda").mul(0.05) if r["bias"] else None
    r["bias"] = bias.double().cpu().numpy() if bias is not None else None
    router = make(ctx, r)
    w, idx = run(router, logits, bias)
    l = logits.double().cpu().numpy()
    s, v = values64(l, r)
    got, weights = idx.cpu().numpy().astype(np.int64), w.double().cpu().numpy()
    assert got.min() >= 0 and got.max() < E
    assert all(len(set(row)) == k for row in got)
    best = -np.sort(-v, -1)[:, :k]
    chosen = np.take_along_axis(v, got, -1)
    np.testing.assert_allclose(chosen, best, rtol=2.0 ** -21, atol=2.0 ** -22)
    want = np.take_along_axis(s, got, -1)
    if r["renormalize"]:
        want = want / (want.sum(-1, keepdims=True) + 1e-20)
    np.testing.assert_allclose(weights, want * r["scale"], rtol=64 * 2.0 ** -23, atol=1e-30)


def test_ties_and_special_values(ctx):
    """Equal values: the lowest index.  NaN and -infinity last, in index order.  Exact for logits as the choice's values."""
    inf, nan = float("inf"), float("nan")
    rows = [
        [0.0, -0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0],
        [1.0, 3.0, 3.0, 2.0, 3.0, 1.0, 1.0, 0.0],
        [-inf, -inf, 5.0, -inf, -inf, -inf, -inf, -inf],
        [nan, 1.0, nan, 0.0, -inf, nan, nan, nan],
        [-1.0, -1.0, -2.0, -0.5, -3.0, -0.5, -9.0, -9.0],
    ]
    want = [[0, 1, 2, 3], [1, 2, 4, 3], [2, 0, 1, 3], [1, 3, 0, 2], [3, 5, 0, 1]]
    w, i = run(routing.Router(ctx, 8, 4, score="softmax"), torch.tensor(rows, device="cuda"))
    assert i.tolist() == want
    assert torch.equal(w[0], torch.full((4,), 0.25, device="cuda")) and w[2].tolist() == [1.0, 0.0, 0.0, 0.0]
    # all -infinity: no score at all, weights 0 and the first experts
    w, i = run(routing.Router(ctx, 40, 3, score="softmax"), torch.full((2, 40), -inf, device="cuda"))
    assert i.tolist() == [[0, 1, 2]] * 2 and bool((w == 0).all())
    w, i = run(routing.Router(ctx, 40, 3, score="sigmoid"), torch.full((2, 40), -inf, device="cuda"))
    assert i.tolist() == [[0, 1, 2]] * 2 and bool((w == 0).all())
    # experts of groups that are left out count as -infinity: they follow, in index order, only where nothing else is left
    logits = torch.zeros(1, 8, device="cuda")
    logits[0, 4:] = 1.0
    logits[0, 5:] = -inf
    _, i = run(routing.Router(ctx, 8, 4, score="softmax", groups=2, top_groups=1), logits)
    assert i[0, 0] == 4 and i[0, 1:].tolist() == [0, 1, 2]


@pytest.mark.parametrize("count", [0, 1, 31, 264, 1024, 4097, 40000, 131072])
@pytest.mark.parametrize("experts", [1, 7, 64, 512])
def test_sort(ctx, count, experts):
    g = torch.Generator(device="cuda").manual_seed(count + experts)
    idx = torch.randint(0, experts, (count,), generator=g, device="cuda", dtype=torch.int32)
    if count > 100:
        idx[idx == experts // 2] = 0                          # an expert without tokens (for one expert: itself)
        idx[::17] = -1                                        # choices of no expert
        idx[5] = experts
    router = routing.Router(ctx, experts, 1)
    offsets = torch.full((experts + 1,), -9, dtype=torch.int32, device="cuda")
    order, position = (torch.full((count,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    router.sort(idx, offsets, order, position)
    i = idx.cpu().numpy().astype(np.int64)
    valid = np.flatnonzero((i >= 0) & (i < experts))
    want = valid[np.argsort(i[valid], kind="stable")]
    ends = np.concatenate([[0], np.cumsum(np.bincount(i[valid], minlength=experts))])
    assert offsets.tolist() == ends.tolist()
    got = order.cpu().numpy()
    assert np.array_equal(got[:len(want)], want) and (got[len(want):] == -1).all()
    pos = np.full(count, -1)
    pos[want] = np.arange(len(want))
    assert np.array_equal(position.cpu().numpy(), pos)


@pytest.mark.parametrize("count", [1000, 100003])
def test_sort_as_many_experts_as_the_library_takes(ctx, count):
    """1024 experts (a router has 512 at most), one cluster's shared memory nearly full."""
    experts = 1024
    g = torch.Generator(device="cuda").manual_seed(count)
    idx = torch.randint(-1, experts + 1, (count,), generator=g, device="cuda", dtype=torch.int32)
    offsets = torch.full((experts + 1,), -9, dtype=torch.int32, device="cuda")
    order, position = (torch.full((count,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    L = routing.lib()
    stream = torch.cuda.current_stream().cuda_stream
    assert L.hgemm_route_sort(ctx._h, idx.data_ptr(), count, experts, offsets.data_ptr(), order.data_ptr(), position.data_ptr(), stream) == hgemm.OK
    i = idx.cpu().numpy().astype(np.int64)
    valid = np.flatnonzero((i >= 0) & (i < experts))
    want = valid[np.argsort(i[valid], kind="stable")]
    assert offsets.tolist() == np.concatenate([[0], np.cumsum(np.bincount(i[valid], minlength=experts))]).tolist()
    got = order.cpu().numpy()
    assert np.array_equal(got[:len(want)], want) and (got[len(want):] == -1).all()
    pos = np.full(count, -1)
    pos[want] = np.arange(len(want))
    assert np.array_equal(position.cpu().numpy(), pos)
    assert L.hgemm_route_sort(ctx._h, idx.data_ptr(), count, experts + 1, offsets.data_ptr(), order.data_ptr(), position.data_ptr(), stream) == hgemm.ERR_INVALID_ARG


def loss64(l, idx, dw, r):
    s = scores64(l, r["score"])
    w = np.take_along_axis(s, idx, -1)
    if r["renormalize"]:
        w = w / (w.sum(-1, keepdims=True) + 1e-20)
    return (w * r["scale"] * dw).sum(-1)


@pytest.mark.parametrize("t", RULES, ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_gradient(ctx, t, dtype):
    """Against the formula in 64 bits: 32-bit sums of at most 32 terms whose magnitudes are bounded by scale * max |dw| (over the
    smallest sum of chosen scores where weights are renormalised), then the type's own rounding.  And against differences."""
    r = rule(t)
    r["bias"] = None
    E, k, T = r["experts"], r["top_k"], 37
    g = torch.Generator(device="cuda").manual_seed(E)
    logits = torch.randn(T, E, generator=g, device="cuda").mul(2.0).to(dtype)
    idx = torch.stack([torch.randperm(E, generator=g, device="cuda")[:k] for _ in range(T)]).int()
    dw = torch.randn(T, k, generator=g, device="cuda")
    dl = torch.full((T, E + 5), float("nan"), dtype=dtype, device="cuda")
    make(ctx, r).backward(logits, idx, dw, dl[:, :E])
    assert bool(torch.isnan(dl[:, E:]).all())
    got = dl[:, :E].double().cpu().numpy()
    l, i, d = logits.double().cpu().numpy(), idx.cpu().numpy().astype(np.int64), dw.double().cpu().numpy()
    s = scores64(l, r["score"])
    c = np.take_along_axis(s, i, -1)
    total = c.sum(-1, keepdims=True) + 1e-20
    dc = d * r["scale"]
    if r["renormalize"]:
        dc = (dc - (dc * c).sum(-1, keepdims=True) / total) / total
    ds = np.zeros_like(s)
    np.put_along_axis(ds, i, dc, -1)
    want = ds * s * (1 - s) if r["score"] == "sigmoid" else s * (ds - (s * ds).sum(-1, keepdims=True))
    size = np.abs(d * r["scale"]).max(-1, keepdims=True) * (1.0 / total if r["renormalize"] else 1.0)
    unit = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype]
    tiny = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}[dtype]
    bound = 128 * 2.0 ** -24 * size * (s + 2.0 ** -24) + unit * np.abs(want) + tiny
    assert (np.abs(got - want) <= bound).all()
    if dtype == torch.float32:
        h = 1e-5
        for e in {0, E // 2, E - 1, int(i[0, 0])}:
            up, down = l.copy(), l.copy()
            up[:, e] += h
            down[:, e] -= h
            slope = (loss64(up, i, d, r) - loss64(down, i, d, r)) / (2 * h)
            # the difference's own error: h^2 of the third derivative and 64-bit cancellation over h
            np.testing.assert_allclose(got[:, e], slope, atol=float((bound[:, e] + 1e-8 * size[:, 0]).max()), rtol=0)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_gradient_of_one_renormalised_choice_is_zero(ctx, score, dtype):
    """s / (s + 1e-20) is 1 in 32 bits for every s above 2^24 * 1e-20 (the logits here keep s above 1e-12), so the weight does not
    depend on the logits: its gradient is exactly zero."""
    T, E = 1000, 60
    g = torch.Generator(device="cuda").manual_seed(11)
    logits = torch.randn(T, E, generator=g, device="cuda").mul(3.0).clamp(-9, 9).to(dtype)
    router = routing.Router(ctx, E, 1, score=score, renormalize=True, scale=2.5)
    w, i = run(router, logits)
    assert bool((w == 2.5).all())
    for idx in (i, torch.randint(0, E, (T, 1), generator=g, device="cuda", dtype=torch.int32)):
        dl = torch.full_like(logits, float("nan"))
        router.backward(logits, idx, torch.randn(T, 1, generator=g, device="cuda") * 100.0, dl)
        assert bool((dl == 0).all())


def test_same_bits_every_time(ctx):
    g = torch.Generator(device="cuda").manual_seed(3)
    logits = torch.randn(5000, 256, generator=g, device="cuda")
    router = routing.Router(ctx, 256, 8, score="sigmoid", groups=8, top_groups=4, group_score="top2")
    first = None
    for _ in range(4):
        w, i = run(router, logits)
        out = [torch.empty(257, dtype=torch.int32, device="cuda"), torch.empty(40000, dtype=torch.int32, device="cuda"), torch.empty(40000, dtype=torch.int32, device="cuda")]
        router.sort(i, *out)
        now = [w, i, *out]
        first = first or now
        assert all(torch.equal(a, b) for a, b in zip(first, now))


def test_no_tokens(ctx):
    router = routing.Router(ctx, 16, 2)
    empty = lambda *s, **k: torch.empty(*s, device="cuda", **k)  # noqa: E731
    router.forward(empty(0, 16), empty(0, 2), empty(0, 2, dtype=torch.int32))
    router.backward(empty(0, 16), empty(0, 2, dtype=torch.int32), empty(0, 2), empty(0, 16))
    torch.cuda.synchronize()


def test_refusals(ctx):
    Router = routing.Router
    for kw in (dict(experts=0, top_k=1), dict(experts=513, top_k=1), dict(experts=8, top_k=9), dict(experts=64, top_k=33), dict(experts=8, top_k=0),
               dict(experts=8, top_k=1, groups=3), dict(experts=8, top_k=1, groups=4, top_groups=5), dict(experts=8, top_k=3, groups=4, top_groups=1),
               dict(experts=8, top_k=1, groups=8, top_groups=2, group_score="top2", score="sigmoid"), dict(experts=8, top_k=1, scale=float("nan"))):
        with pytest.raises(hgemm.HgemmError):
            Router(ctx, **kw)
    with pytest.raises(ValueError):
        Router(ctx, 8, 1, score="tanh")
    r = Router(ctx, 8, 2)
    l, w, i = torch.zeros(5, 8, device="cuda"), torch.full((5, 2), 3.0, device="cuda"), torch.zeros(5, 2, dtype=torch.int32, device="cuda")
    for call in (lambda: r.forward(l[:, :7], w, i), lambda: r.forward(l.double(), w, i), lambda: r.forward(l, w[:4], i), lambda: r.forward(l, w, i.long()),
                 lambda: r.forward(l, w, i, bias=torch.zeros(7, device="cuda")), lambda: r.forward(l.t().contiguous().t(), w, i),
                 lambda: r.backward(l, i, w, l.half()), lambda: r.sort(i, torch.zeros(8, dtype=torch.int32, device="cuda"), i.flatten(), i.flatten())):
        with pytest.raises(ValueError):
            call()
    # the two best softmax scores of a group need scores, not logits: only with a bias
    two = Router(ctx, 8, 2, groups=2, top_groups=1, group_score="top2")
    with pytest.raises(hgemm.HgemmError):
        two.forward(l, w, i)
    two.forward(l, w.clone(), i, bias=torch.zeros(8, device="cuda"))
    torch.cuda.synchronize()
    assert bool((w == 3.0).all())
