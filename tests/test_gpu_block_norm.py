"""kan_block_norm_forward / kan_block_norm_backward against their definitions in 64 bits."""
import pytest

from tokens_testlib import check, norms, norms_grad

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def kb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2512_15742_amd import binding
    binding.lib()
    return binding


def draw(seed, N, D, stream, block, weight, gate=True, first=False, bare=False):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, type, mul=1.0, add=0.0):
        return (torch.randn(shape, generator=g, device="cuda") * mul + add).to(type)
    return dict(x=normal(N, D, type=stream, mul=2.0), v=None if first else normal(N, D, type=block, mul=0.7),
                gate=normal(N, D, type=block, mul=3.0) if gate and not first else None,
                wa=None if first or bare else normal(D, type=weight, mul=0.2, add=1.0), wb=None if bare else normal(D, type=weight, mul=0.1, add=0.3),
                dy=normal(N, D, type=stream), du=normal(N, D, type=block))


SHAPES = [
    (1, 1, F32, F32, F32), (1, 2048, BF16, F32, BF16), (3, 7, F16, F16, F32), (5, 64, BF16, BF16, BF16), (130, 500, F32, F32, F32),
    (130, 513, F16, F32, F16), (37, 1000, F32, F32, BF16), (999, 1025, BF16, BF16, F32), (600, 2047, BF16, F32, BF16), (515, 2049, F16, F16, F16),
    (20, 4096, BF16, BF16, BF16), (700, 4097, F32, F32, F32), (9, 8192, BF16, F32, F32), (6, 8193, F32, F32, F32), (3, 16384, BF16, BF16, BF16),
    (3, 16383, F16, F32, F16), (5000, 96, BF16, F32, BF16),
]


@pytest.mark.parametrize("N,D,stream,block,weight", SHAPES)
@pytest.mark.parametrize("form", ["gated", "plain", "first", "last", "bare"])
def test_both_directions(kb, N, D, stream, block, weight, form):
    t = draw(N * 7 + D, N, D, stream, block, weight, gate=form == "gated", first=form == "first", bare=form == "bare")
    scale, eps = 0.75, 1e-5
    y, u = kb.kan_block_norm_forward(t["x"], v=t["v"], gate=t["gate"], w_after=t["wa"], w_before=None if form == "last" else t["wb"], scale=scale,
                                     eps=eps, dtype=block, want_u=form != "last")
    ry, ey, ru, eu = norms(t["x"], t["v"], t["gate"], t["wa"], t["wb"], scale, eps)
    if form == "first":
        assert y is None
    else:
        assert y.dtype == stream
        check(y, ry, ey)
    if form == "last":
        assert u is None
    else:
        assert u.dtype == block
        check(u, ru, eu)
    du = None if form == "last" else t["du"]
    dy = None if form == "plain" else t["dy"]
    args = dict(dy=dy, du=du, v=t["v"], gate=t["gate"], w_after=t["wa"], w_before=t["wb"], scale=scale, eps=eps)
    if dy is None and du is None:
        return
    got = kb.kan_block_norm_backward(t["x"], **args)
    refs = norms_grad(t["x"], dy, du, t["v"], t["gate"], t["wa"], t["wb"], scale, eps)
    for a, r, name in zip(got, refs, ("dx", "dv", "dgate", "dw_before", "dw_after")):
        assert (a is None) == (r is None), name
        if a is not None:
            check(a, *r)
    again = kb.kan_block_norm_backward(t["x"], **args)
    assert all((a is None and b is None) or torch.equal(a, b) for a, b in zip(got, again))


def test_gradients_are_differences(kb):
    """Directional derivative of sum(y dy) + sum(u du) in fp32 against the gradients: the central difference's own error is
    of the third order of the step, 2^-7, its roundings 2^-24 over 2^-6 of sums of some 600 terms of order one."""
    t = draw(3, 6, 50, F32, F32, F32)
    names = ("x", "v", "gate", "wa", "wb")
    step = {k: torch.randn(t[k].shape, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda") for i, k in enumerate(names)}

    def value(s):
        a = {k: t[k] + s * step[k] for k in names}
        y, u = kb.kan_block_norm_forward(a["x"], v=a["v"], gate=a["gate"], w_after=a["wa"], w_before=a["wb"], scale=0.5)
        return float((y.double() * t["dy"].double()).sum() + (u.double() * t["du"].double()).sum())
    y, _ = kb.kan_block_norm_forward(t["x"], v=t["v"], gate=t["gate"], w_after=t["wa"], w_before=t["wb"], scale=0.5)
    got = kb.kan_block_norm_backward(y, dy=t["dy"], du=t["du"], v=t["v"], gate=t["gate"], w_after=t["wa"], w_before=t["wb"], scale=0.5)
    along = sum(float((g.double() * step[k].double()).sum()) for g, k in zip((got[0], got[1], got[2], got[4], got[3]), names))
    h = 2.0 ** -7
    diff = (value(h) - value(-h)) / (2 * h)
    third = abs((value(2 * h) - value(-2 * h)) / (4 * h) - diff)       # three times the leading error of the difference at h
    assert abs(along - diff) <= third + 600 * 8 * 2.0 ** -24 * 64, (along, diff, third)


def test_zero_rows_and_rows_of_no_numbers(kb):
    t = draw(8, 6, 300, F32, F32, F32)
    t["x"][0] = 0.0
    t["v"][0] = 0.0
    t["v"][1] = 0.0
    t["x"][2] = float("nan")
    t["v"][3, 5] = float("inf")
    t["gate"][4] = -200.0
    t["gate"][5] = 200.0
    y, u = kb.kan_block_norm_forward(t["x"], v=t["v"], gate=t["gate"], w_after=t["wa"], w_before=t["wb"])
    assert not y[0].any() and not u[0].any() and torch.equal(y[1], t["x"][1])
    assert bool(y[2].isnan().all()) and bool(u[2].isnan().all()) and bool(y[3, 5].isnan())
    assert torch.equal(y[4], t["x"][4])
    ry, ey, ru, eu = norms(t["x"], t["v"], t["gate"], t["wa"], t["wb"], 1.0, 1e-6)
    check(y[4:], ry[4:], ey[4:])
    check(u[4:], ru[4:], eu[4:])
    got = kb.kan_block_norm_backward(t["x"], dy=t["dy"], du=t["du"], v=t["v"], gate=t["gate"], w_after=t["wa"], w_before=t["wb"])
    refs = norms_grad(t["x"], t["dy"], t["du"], t["v"], t["gate"], t["wa"], t["wb"], 1.0, 1e-6)
    for a, r in zip(got[:3], refs[:3]):
        for rows in (slice(0, 2), slice(4, 6)):
            check(a[rows], r[0][rows], r[1][rows])


def test_in_place_and_between_others(kb):
    """y over x, dx over dy (C-ABI), outputs that start off a 16-byte boundary between others."""
    import ctypes as C
    N, D = 37, 333
    t = draw(21, N, D, BF16, F32, F32)
    args = dict(v=t["v"], gate=t["gate"], w_after=t["wa"], w_before=t["wb"], scale=0.5)
    y, u = kb.kan_block_norm_forward(t["x"], **args)
    whole_y = torch.full((N * D + 9,), 7.0, dtype=BF16, device="cuda")
    whole_u = torch.full((N * D + 9,), 7.0, device="cuda")
    yi, ui = whole_y[3:3 + N * D].view(N, D).copy_(t["x"]), whole_u[5:5 + N * D].view(N, D)
    y2, u2 = kb.kan_block_norm_forward(yi, y=yi, u=ui, **args)
    assert y2.data_ptr() == yi.data_ptr() and torch.equal(yi, y) and torch.equal(ui, u)
    assert bool((whole_y[:3] == 7).all() & (whole_y[3 + N * D:] == 7).all() & (whole_u[:5] == 7).all() & (whole_u[5 + N * D:] == 7).all())
    got = kb.kan_block_norm_backward(y, dy=t["dy"], du=t["du"], **args)
    b = kb.kan_block_norm(D, kb.KAN_BF16, kb.KAN_F32, kb.KAN_F32, t["wb"].data_ptr(), t["wa"].data_ptr(), 0.5, 1e-6)
    dx, dv, dg = t["dy"].clone(), torch.empty_like(t["v"]), torch.empty_like(t["v"])
    p = lambda a: C.c_void_p(a.data_ptr())      # noqa: E731
    st = kb.lib().kan_block_norm_backward(C.byref(b), p(y), p(dx), p(t["du"]), p(t["v"]), p(t["gate"]), N, p(dx), p(dv), p(dg), None, None, None, 0,
                                          C.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert st == kb.KAN_OK
    assert torch.equal(dx, got[0]) and torch.equal(dv, got[1]) and torch.equal(dg, got[2])


def test_no_rows(kb):
    t = draw(1, 0, 40, BF16, F32, F32)
    y, u = kb.kan_block_norm_forward(t["x"], v=t["v"], gate=t["gate"], w_after=t["wa"], w_before=t["wb"])
    assert y.shape == (0, 40) and u.shape == (0, 40)
    got = kb.kan_block_norm_backward(t["x"], dy=t["dy"], du=t["du"], v=t["v"], gate=t["gate"], w_after=t["wa"], w_before=t["wb"])
    assert not got[3].any() and not got[4].any()


def test_replays_from_a_graph(kb):
    sets = [draw(s, 700, 1000, BF16, F32, F32) for s in range(4)]
    keys = ("x", "v", "gate", "dy", "du")

    def run(t):
        y, u = kb.kan_block_norm_forward(t["x"], v=t["v"], gate=t["gate"], w_after=sets[0]["wa"], w_before=sets[0]["wb"])
        return (y, u) + kb.kan_block_norm_backward(y, dy=t["dy"], du=t["du"], v=t["v"], gate=t["gate"], w_after=sets[0]["wa"], w_before=sets[0]["wb"])
    eager = [run(t) for t in sets]
    held = {k: sets[0][k].clone() for k in keys}
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            out = run(held)
    for k in (2, 1, 3, 0, 1):
        for name in keys:
            held[name].copy_(sets[k][name])
        for o in out:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager[k]))
