"""kan_block_norm_forward / kan_block_norm_backward where rows, streams and gates are at the ends of their ranges, against
their definitions in 64 bits."""
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


def draw(seed, N, D, stream, block, weight):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, type, mul=1.0, add=0.0):
        return (torch.randn(shape, generator=g, device="cuda") * mul + add).to(type)
    return dict(x=normal(N, D, type=stream, mul=2.0), v=normal(N, D, type=block, mul=0.7), gate=normal(N, D, type=block, mul=3.0),
                wa=normal(D, type=weight, mul=0.2, add=1.0), wb=normal(D, type=weight, mul=0.1, add=0.3), dy=normal(N, D, type=stream),
                du=normal(N, D, type=block))


@pytest.mark.parametrize("stream,block,weight", [(F32, F32, F32), (BF16, BF16, F32), (F16, F32, F16)])
@pytest.mark.parametrize("D", [1, 2, 3, 4, 5, 6, 7])
def test_rows_of_fewer_than_eight_columns(kb, D, stream, block, weight):
    """The last rows of an array share eight elements with the rows in front of them, which hold nothing of theirs."""
    for N in range(2, 18):
        t = draw(100 * D + N, N, D, stream, block, weight)
        scale, eps = 0.75, 1e-5
        y, u = kb.kan_block_norm_forward(t["x"], v=t["v"], gate=t["gate"], w_after=t["wa"], w_before=t["wb"], scale=scale, eps=eps)
        ry, ey, ru, eu = norms(t["x"], t["v"], t["gate"], t["wa"], t["wb"], scale, eps)
        check(y, ry, ey)
        check(u, ru, eu)
        _, first = kb.kan_block_norm_forward(t["x"], w_before=t["wb"], eps=eps, dtype=block)
        check(first, *norms(t["x"], None, None, None, t["wb"], scale, eps)[2:])
        got = kb.kan_block_norm_backward(t["x"], dy=t["dy"], du=t["du"], v=t["v"], gate=t["gate"], w_after=t["wa"], w_before=t["wb"], scale=scale, eps=eps)
        for a, r in zip(got, norms_grad(t["x"], t["dy"], t["du"], t["v"], t["gate"], t["wa"], t["wb"], scale, eps)):
            check(a, *r)


@pytest.mark.parametrize("form", ["first", "last", "both"])
def test_streams_of_more_rows_than_workgroups(kb, form):
    """More than 2^20 rows of several waves each: a workgroup takes further rows, with one sum a row or two."""
    N, D, part = 2 ** 20 + 3 * 2 ** 15 + 77, 1032, 2 ** 15
    g = torch.Generator(device="cuda").manual_seed(31)
    x = torch.empty((N, D), dtype=BF16, device="cuda")
    for n in range(0, N, part):
        x[n:n + part] = torch.randn((min(part, N - n), D), generator=g, device="cuda") * (0.25 + torch.rand((min(part, N - n), 1), generator=g, device="cuda"))
    v = None if form == "first" else x.flip(0)
    wb = (torch.randn(D, generator=g, device="cuda") * 0.1 + 0.3) if form != "last" else None
    args = dict(v=v, w_before=wb, scale=0.5, eps=1e-5, want_u=form != "last")
    y, u = kb.kan_block_norm_forward(x, **args)
    for n in [*range(0, N - 2 ** 20, part // 4), 2 ** 19, *range(2 ** 20 - part // 4, N, part // 4)]:      # rows of workgroups with two of them, and others
        rows = slice(n, min(N, n + part // 4))
        ry, ey, ru, eu = norms(x[rows], None if v is None else v[rows], None, None, wb, 0.5, 1e-5)
        if y is not None:
            check(y[rows], ry, ey)
        if u is not None:
            check(u[rows], ru, eu)
    again = kb.kan_block_norm_forward(x, **args)
    assert all(a is None or torch.equal(a, b) for a, b in zip((y, u), again))


def test_gradient_of_gates_far_from_zero(kb):
    """dgate goes with sigma(z) sigma(-z): as exact for open gates, where 1 - sigma is a difference of nearly equal numbers, as for
    closed ones.  Its bound is norms_grad's (a quotient of the exponential is off by up to |z| half steps, the sums by 128), in terms of
    the whole product."""
    N, D = 22, 96
    t = draw(41, N, D, F32, F32, F32)
    z = torch.tensor([5.0, 8, 10, 12, 14, 16, 17, 18, 20, 25, 30], device="cuda")
    t["gate"] = (torch.cat([z, -z])[:, None] + torch.linspace(0, 0.5, D, device="cuda")).contiguous()
    got = kb.kan_block_norm_backward(t["x"], dy=t["dy"], du=t["du"], v=t["v"], gate=t["gate"], w_after=t["wa"], w_before=t["wb"], scale=0.5)
    ref, bound = norms_grad(t["x"], t["dy"], t["du"], t["v"], t["gate"], t["wa"], t["wb"], 0.5, 1e-6)[2]
    zd = t["gate"].double()
    other = torch.sigmoid(-zd)
    check(got[2], ref / (1 - torch.sigmoid(zd)) * other, bound * other)


def test_sums_of_the_groups_are_trees(kb):
    """Rows of ones: a term of dw_before is an entry of du, exact, and only its sum over 512 rows, one a group, is rounded.  A
    rounding is off by at most U of its value, evenly: a level of a tree with n sums of S / n adds S^2 U^2 / (3 n) to the mean square,
    all levels 2/3 S^2 U^2 at most (64 sums one behind the other: up to 64/9 S^2 U^2)."""
    N, D = 512, 2048
    y = torch.ones((N, D), device="cuda")
    du = torch.rand((N, D), generator=torch.Generator(device="cuda").manual_seed(51), device="cuda") + 1.0
    got = kb.kan_block_norm_backward(y, du=du, w_before=torch.ones(D, device="cuda"), eps=1e-12)[3]
    ref = du.double().sum(0)
    assert float(((got.double() - ref) / ref).square().mean().sqrt()) <= (2 / 3) ** 0.5 * 2.0 ** -24
