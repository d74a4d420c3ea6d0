"""kan_vocab_loss_forward / kan_vocab_loss_backward against their definitions in 64 bits."""
import pytest

from tokens_testlib import Loss, check, check_rms

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


def draw(seed, N, V, D, dtype, kind="i64", left_out=0.2, spread=2.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    table = (torch.randn((V, D), generator=g, device="cuda") * (spread / D ** 0.5)).to(dtype)
    t = torch.randint(0, V, (N,), generator=g, device="cuda")
    none = torch.rand(N, generator=g, device="cuda") < left_out
    h = torch.randn((N, D), generator=g, device="cuda") + 2 * torch.rand((N, 1), generator=g, device="cuda") * table[t].float()
    if kind == "u16":
        t = torch.where(none & (V < 65536), 65535, t)
        t = torch.where(t >= 32768, t - 65536, t).to(torch.int16)
    elif kind == "i32":
        t = torch.where(none, -1, t).to(torch.int32)
    else:
        t = torch.where(none, torch.where(t % 2 == 0, -100, V), t)
    dloss = torch.randn(N, generator=g, device="cuda") / N
    return h.to(dtype), table, t, dloss


def check_all(kb, h, table, t, dloss, scale):
    loss, lse = kb.kan_vocab_loss_forward(h, table, t, scale=scale)
    ref = Loss(h, table, t, scale)
    check(lse, ref.lse, ref.elog)
    check(loss, ref.loss, ref.eloss)
    assert not loss[~ref.ok].any()
    dh, dt = kb.kan_vocab_loss_backward(h, table, t, lse, dloss, scale=scale)
    assert dh.dtype == h.dtype and dt.dtype == h.dtype
    for got, (want, bound, deviation) in zip((dh, dt), ref.grads(dloss)):
        check(got, want, bound)
        check_rms(got, want, deviation)
    assert not dh[~ref.ok].any()
    again = kb.kan_vocab_loss_backward(h, table, t, lse, dloss, scale=scale)
    assert torch.equal(again[0], dh) and torch.equal(again[1], dt)
    assert all(torch.equal(a, b) for a, b in zip(kb.kan_vocab_loss_forward(h, table, t, scale=scale), (loss, lse)))
    return loss, lse, dh, dt


SIZES = [
    (1, 1, 1), (1, 2, 8), (1, 65536, 64), (2, 300, 7), (5, 129, 1000), (15, 5000, 256), (16, 4097, 96), (17, 1000, 65), (64, 1111, 512), (65, 255, 33),
    (128, 256, 128), (129, 257, 129), (255, 3001, 72), (300, 513, 640), (511, 20000, 40), (700, 1500, 2048), (1030, 2050, 136),
]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("N,V,D", SIZES)
def test_both_directions(kb, N, V, D, dtype):
    kind = ("i64", "i32", "u16")[(N + D) % 3]
    check_all(kb, *draw(N + V + D, N, V, D, dtype, kind), scale=(1.0, 0.5)[N % 2])


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("N,V,D", [(5000, 3001, 72), (4097, 16500, 264), (1500, 9000, 1032)])
def test_many_tokens(kb, N, V, D, dtype):
    """Large tiles, long and short contractions, more tokens than a workgroup counts by itself."""
    check_all(kb, *draw(N + D, N, V, D, dtype, ("i32", "i64", "u16")[N % 3]), scale=1.0)


@pytest.mark.parametrize("N,V,D", [(1, 31, 3), (3, 1000, 70), (31, 33, 129), (32, 2085, 64), (33, 100, 250), (60, 1200001, 12), (63, 4999, 300)])
def test_few_tokens_in_full_precision(kb, N, V, D):
    check_all(kb, *draw(N + D, N, V, D, F32, ("i32", "i64")[N % 2]), scale=0.5)


@pytest.mark.parametrize("dtype,N,V,D", [(F16, 40, 50001, 1000), (BF16, 2500, 132000, 64), (F32, 300, 150001, 200)])
def test_tables_in_several_pieces(kb, dtype, N, V, D):
    check_all(kb, *draw(1, N, V, D, dtype), scale=1.0)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_added_onto_a_table(kb, dtype):
    """The table's gradient on top of another one, outputs between others."""
    h, table, t, dloss = draw(4, 200, 999, 88, dtype)
    loss, lse = kb.kan_vocab_loss_forward(h, table, t)
    n = table.numel()
    whole = torch.full((n + 64,), float("nan"), dtype=dtype, device="cuda")
    base = whole[8:8 + n].view(table.shape)
    old = (torch.randn(table.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)) * 0.01).to(dtype)
    base.copy_(old)
    whole_h = torch.full((h.numel() + 64,), float("nan"), dtype=dtype, device="cuda")
    dh = whole_h[8:8 + h.numel()].view(h.shape)
    kb.kan_vocab_loss_backward(h, table, t, lse, dloss, dh=dh, dtable=base, accumulate=True)
    (want_h, bh, _), (want, bound, _) = Loss(h, table, t, 1.0).grads(dloss)
    check(base, want + old.double(), bound + 2.0 ** -24 * (want + old.double()).abs())
    check(dh, want_h, bh)
    assert bool(whole[:8].isnan().all() & whole[8 + n:].isnan().all())
    assert bool(whole_h[:8].isnan().all() & whole_h[8 + h.numel():].isnan().all())


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_rows_that_are_left_out_hold_anything(kb, dtype):
    h, table, t, dloss = draw(6, 300, 700, 120, dtype, left_out=0.4)
    out = (t < 0) | (t >= 700)
    clean_loss, clean_lse = kb.kan_vocab_loss_forward(h, table, t)
    clean = kb.kan_vocab_loss_backward(h, table, t, clean_lse, dloss)
    bad = h.clone()
    bad[out] = float("nan")
    bad[out.nonzero()[0, 0]] = float("inf")
    dl = torch.where(out, float("nan"), dloss)
    loss, lse = kb.kan_vocab_loss_forward(bad, table, t)
    assert torch.equal(loss, clean_loss) and torch.equal(lse[~out], clean_lse[~out])
    lse = torch.where(out, float("nan"), lse)
    got = kb.kan_vocab_loss_backward(bad, table, t, lse, dl)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    # none is left: no loss, no gradient
    none = torch.full_like(t, -1)
    loss, lse = kb.kan_vocab_loss_forward(h, table, none)
    assert not loss.any()
    for g in kb.kan_vocab_loss_backward(h, table, none, lse, dloss):
        assert not g.any()


def test_logits_far_apart(kb):
    """Logits of thousands, of which the target's is the largest, the smallest, or behind a tile of far smaller ones."""
    N, V, D = 40, 777, 16
    table = torch.zeros((V, D), device="cuda")
    table[:, 0] = torch.linspace(-60, 60, V, device="cuda")
    h = torch.zeros((N, D), device="cuda")
    h[:, 0] = torch.linspace(-90, 90, N, device="cuda")
    t = torch.arange(N, device="cuda") % 3 * (V // 2)
    for dtype in (BF16, F16, F32):
        check_all(kb, h.to(dtype), table.to(dtype), t, torch.full((N,), 0.25, device="cuda"), scale=1.0)
        check_all(kb, h.to(dtype), table.to(dtype), t, torch.full((N,), 0.25, device="cuda"), scale=-2.0)
    # every logit far below 0 in the only tile that has rows: nothing underflows
    loss, lse = kb.kan_vocab_loss_forward(torch.full((3, D), -100.0, device="cuda"), torch.full((5, D), 10.0, device="cuda"), torch.zeros(3, dtype=torch.long, device="cuda"))
    assert bool(((lse + 16000 - 1.6094379).abs() < 16000 * 2.0 ** -22).all())


def test_values_that_are_no_numbers_stay_in_their_rows(kb):
    h, table, t, dloss = draw(8, 50, 300, 64, BF16, left_out=0.0)
    clean = kb.kan_vocab_loss_forward(h, table, t)
    h[3, 5] = float("nan")
    loss, lse = kb.kan_vocab_loss_forward(h, table, t)
    keep = torch.arange(50, device="cuda") != 3
    assert bool(loss[3].isnan()) and bool(lse[3].isnan())
    assert torch.equal(loss[keep], clean[0][keep]) and torch.equal(lse[keep], clean[1][keep])
    z = torch.zeros((2, 8), dtype=BF16, device="cuda")
    z[0, 0], z[1, 0] = float("inf"), 1.0
    w = torch.zeros((20, 8), dtype=BF16, device="cuda")
    w[:, 0] = 1.0
    loss, lse = kb.kan_vocab_loss_forward(z, w, torch.zeros(2, dtype=torch.long, device="cuda"))
    assert float(lse[0]) == float("inf") and abs(float(lse[1]) - 1 - 2.9957323) < 1e-5


def test_half_gradients_of_small_and_of_scaled_losses(kb):
    """fp16: gradients of losses that are scaled up to keep them out of the subnormals, and of ones that are not."""
    for mul in (1.0, 65536.0 / 64):
        h, table, t, dloss = draw(12, 333, 5000, 64, F16)
        check_all(kb, h, table, t, dloss.sign() / 333 * mul, scale=1.0)
    _, lse = kb.kan_vocab_loss_forward(h, table, t)
    for mul in (0.0, 1e-36, 1e-44):               # gradients below the smallest number of fp16: zeros
        for g in kb.kan_vocab_loss_backward(h, table, t, lse, dloss.sign() * mul):
            assert not g.any()


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("N", [255, 255 * 32])
def test_gradients_of_a_mean_are_not_all_too_large(kb, N, dtype):
    """1 / N is off by 2^-8.01 in bf16.  A target's entry is (p - 1) / N, p at 2^-13 in the mean: off by that in units of 1 / N.  The
    errors of the others and of the results are independent, 2^-8 / sqrt(N D) together at most."""
    g = torch.Generator(device="cuda").manual_seed(21)
    V, D = 8192, 64
    table = (torch.randn((V, D), generator=g, device="cuda") / D ** 0.5).to(dtype)
    h = torch.randn((N, D), generator=g, device="cuda").to(dtype)
    t = torch.randint(0, V, (N,), generator=g, device="cuda")
    dloss = torch.full((N,), 1.0 / N, device="cuda")
    _, lse = kb.kan_vocab_loss_forward(h, table, t)
    for got, (want, _, _) in zip(kb.kan_vocab_loss_backward(h, table, t, lse, dloss), Loss(h, table, t, 1.0).grads(dloss)):
        assert abs(float((got.double() * want).sum() / want.square().sum()) - 1) < 2.0 ** -10


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("N", [70, 4200])
def test_weights_that_are_no_numbers_stay_in_their_rows(kb, N, dtype):
    h, table, t, dloss = draw(22, N, 300, 64, dtype, left_out=0.0)
    _, lse = kb.kan_vocab_loss_forward(h, table, t)
    clean = dloss.clone()
    for row, value in ((3, float("inf")), (5, float("nan")), (N - 1, -float("inf"))):
        clean[row] = 0.0
        dloss[row] = value
    keep = torch.isfinite(dloss)
    dh, _ = kb.kan_vocab_loss_backward(h, table, t, lse, dloss)
    assert torch.equal(dh[keep], kb.kan_vocab_loss_backward(h, table, t, lse, clean)[0][keep])
    assert not torch.isfinite(dh[~keep]).any()


@pytest.mark.parametrize("dtype", [F32])
def test_gradients_are_differences(kb, dtype):
    h, table, t, dloss = draw(14, 30, 200, 24, dtype)
    loss, lse = kb.kan_vocab_loss_forward(h, table, t)
    dh, dt = kb.kan_vocab_loss_backward(h, table, t, lse, dloss)
    g = torch.Generator(device="cuda").manual_seed(1)
    sh, st = torch.randn(h.shape, generator=g, device="cuda"), torch.randn(table.shape, generator=g, device="cuda") / 24 ** 0.5

    def value(s):
        return float((kb.kan_vocab_loss_forward(h + s * sh, table + s * st, t)[0].double() * dloss.double()).sum())
    along = float((dh.double() * sh.double()).sum() + (dt.double() * st.double()).sum())
    step = 2.0 ** -6
    d1, d2 = ((value(s) - value(-s)) / (2 * s) for s in (step, 2 * step))
    # the difference's own error is a third of that between two steps; losses of about 10, weights that sum to about 1
    assert abs(along - d1) <= abs(d2 - d1) + 64 * 10 * 2.0 ** -22, (along, d1, d2)


def test_shapes_and_no_rows(kb):
    h, table, t, dloss = draw(3, 24, 50, 16, F16)
    loss, lse = kb.kan_vocab_loss_forward(h.view(2, 12, 16), table, t.view(2, 12))
    assert loss.shape == (2, 12)
    flat = kb.kan_vocab_loss_forward(h, table, t)
    assert torch.equal(loss.view(-1), flat[0]) and torch.equal(lse.view(-1), flat[1])
    dh, dt = kb.kan_vocab_loss_backward(h.view(2, 12, 16), table, t.view(2, 12), lse, dloss.view(2, 12))
    assert dh.shape == (2, 12, 16)
    none = kb.kan_vocab_loss_forward(h[:0], table, t[:0])
    assert none[0].shape == (0,)
    dh, dt = kb.kan_vocab_loss_backward(h[:0], table, t[:0], none[1], dloss[:0])
    assert dh.shape == (0, 16) and not dt.any()


def test_offsets_past_32_bits(kb):
    """A table of more than 2^32 elements: rows at its end count and get their gradient."""
    V, D, N = 140000, 32768, 3
    table = torch.zeros((V, D), dtype=BF16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    some = torch.tensor([0, 131072, V - 1], device="cuda")
    table[some] = (torch.randn((3, D), generator=g, device="cuda") / 64).to(BF16)
    h = (table[some].float() * 4).to(BF16)
    loss, lse = kb.kan_vocab_loss_forward(h, table, some)
    z = h.double() @ table[some].double().t()
    ref = torch.log(torch.exp(z).sum(1) + (V - 3))
    steps = (D / 4 + 16) * 2.0 ** -24 * float((h.double().abs() @ table[some].double().abs().t()).max())
    check(lse, ref, torch.full_like(ref, steps + 80 * 2.0 ** -24))
    dloss = torch.ones(N, device="cuda")
    dh, dt = kb.kan_vocab_loss_backward(h, table, some, lse, dloss)
    p = torch.exp(z - ref[:, None]) - torch.eye(3, device="cuda")
    want = p.t() @ h.double()
    bound = (p.abs() * 2.0 ** -8 + steps * 4).t() @ h.double().abs()
    check(dt[some], want, bound)
    check(dh, p @ table[some].double(), (p.abs() * 2.0 ** -8 + steps * 4) @ table[some].double().abs())


def test_replays_from_a_graph(kb):
    sets = [draw(s, 200, 3000, 96, BF16) for s in range(4)]

    def run(t):
        loss, lse = kb.kan_vocab_loss_forward(*t[:3])
        return (loss, lse) + kb.kan_vocab_loss_backward(*t[:3], lse, t[3])
    eager = [run(t) for t in sets]
    held = [a.clone() for a in sets[0]]
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            out = run(held)
    for k in (2, 1, 3, 0, 1):
        for a, b in zip(held, sets[k]):
            a.copy_(b)
        for o in out:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager[k]))


def test_two_calls_at_once(kb):
    sets = [draw(s, 150, 2000, 128, F16) for s in range(2)]

    def run(t):
        loss, lse = kb.kan_vocab_loss_forward(*t[:3])
        return (loss, lse) + kb.kan_vocab_loss_backward(*t[:3], lse, t[3])
    alone = [run(t) for t in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(4):
        for k, t in enumerate(sets):
            with torch.cuda.stream(streams[k]):
                got[k].append(run(t))
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(a, b) for r in got[k] for a, b in zip(r, alone[k]))
