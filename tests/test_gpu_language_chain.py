"""A language model of KAN blocks as a program runs it: tokens -> rows of a table -> (norm, KAN head, norm with gate and
residual scale) twice -> norm -> loss against the same table; and the way back, the table's two gradients in one array.
The library has no gradient of KAN layers: the test brings one, and the whole chain is held against automatic
differentiation in 64 bits."""
import numpy as np
import pytest

from paper_2512_15742_amd import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

V, D, HID, N, BLOCKS = 700, 64, 48, 150, 2
EPS, SCALE = 1e-5, 0.5


@pytest.fixture(scope="module")
def kb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2512_15742_amd import binding
    binding.lib()
    return binding


def spline_layer(P, x):
    """A KAN layer (cubic B-spline on seven intervals of [-1, 1], inputs clamped) in 64 bits."""
    book = torch.from_numpy(P.codebook.astype(np.float64) * P.scale).cuda()
    idx = torch.from_numpy(P.idx.astype(np.int64)).cuda()
    c = torch.from_numpy(P.gain.astype(np.float64)).cuda()[..., None] * book[idx] + torch.from_numpy(P.bias.astype(np.float64)).cuda()[..., None]
    p = (x.clamp(-1, 1) + 1) * 3.5
    span = p.detach().floor().clamp(0, 6)
    t = p - span
    w = torch.stack([(1 - t) ** 3, 3 * t ** 3 - 6 * t ** 2 + 4, -3 * t ** 3 + 3 * t ** 2 + 3 * t + 1, t ** 3], -1) / 6      # [n][i][4]
    at = span.long()[..., None] + torch.arange(4, device="cuda")
    basis = torch.zeros((*x.shape, 10), dtype=torch.float64, device="cuda").scatter(-1, at, w)
    return basis.flatten(1) @ c.permute(0, 2, 1).flatten(0, 1)


def block64(Ps, u):
    return spline_layer(Ps[1], torch.tanh(spline_layer(Ps[0], u)))


def model(seed, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s, mul=1.0, add=0.0: (torch.randn(s, generator=g, device="cuda") * mul + add)      # noqa: E731
    m = dict(table=normal(V, D, mul=0.25).to(dtype), w_in=[normal(D, mul=0.02, add=0.2) for _ in range(BLOCKS + 1)],
             w_out=[normal(D, mul=0.1, add=1.0) for _ in range(BLOCKS)], gates=[normal(N, D) for _ in range(BLOCKS)])
    # (the blocks' input norms; the last norm in front of the table is wider)
    m["w_in"][-1] = normal(D, mul=0.1, add=1.0)
    m["params"] = [[synth.make_layer(seed + 10 * b, D, HID, 500), synth.make_layer(seed + 10 * b + 1, HID, D, 500)] for b in range(BLOCKS)]
    ids = torch.randint(0, V, (N,), generator=g, device="cuda")
    targets = torch.where(torch.rand(N, generator=g, device="cuda") < 0.2, -1, torch.randint(0, V, (N,), generator=g, device="cuda"))
    return m, ids, targets


def forward(kb, m, heads, ids, targets):
    """Everything a backward pass needs: streams, block inputs and outputs, rows in front of the loss, losses."""
    ys = [kb.kan_lookup_forward(m["table"], ids, scale=2.0, dtype=torch.float32)]
    us = [kb.kan_block_norm_forward(ys[0], w_before=m["w_in"][0], eps=EPS)[1]]
    vs = []
    for b in range(BLOCKS):
        vs.append(kb.kan_vq_head_forward([heads[b]], us[-1], path=kb.KAN_PATH_GATHER)[0])
        y, u = kb.kan_block_norm_forward(ys[-1], v=vs[-1], gate=m["gates"][b], w_after=m["w_out"][b], w_before=m["w_in"][b + 1], scale=SCALE, eps=EPS)
        ys.append(y)
        us.append(u)
    h = us[-1].to(m["table"].dtype)
    loss, lse = kb.kan_vocab_loss_forward(h, m["table"], targets)
    return ys, us, vs, h, loss, lse


def backward(kb, m, ids, targets, saved, dloss):
    ys, us, vs, h, loss, lse = saved
    dh, dtable = kb.kan_vocab_loss_backward(h, m["table"], targets, lse, dloss)
    du, dy = dh.float(), None
    grads = {"gates": [None] * BLOCKS, "w_in": [None] * (BLOCKS + 1), "w_out": [None] * BLOCKS}
    for b in reversed(range(BLOCKS)):
        dy, dv, grads["gates"][b], grads["w_in"][b + 1], grads["w_out"][b] = kb.kan_block_norm_backward(
            ys[b + 1], dy=dy, du=du, v=vs[b], gate=m["gates"][b], w_after=m["w_out"][b], w_before=m["w_in"][b + 1], scale=SCALE, eps=EPS)
        u = us[b].double().requires_grad_()
        du = torch.autograd.grad(block64(m["params"][b], u), u, dv.double())[0].float()
    dx, _, _, grads["w_in"][0], _ = kb.kan_block_norm_backward(ys[0], dy=dy, du=du, w_before=m["w_in"][0], eps=EPS)
    grads["table"] = kb.kan_lookup_backward(dx, ids, V, scale=2.0, dtable=dtable, accumulate=True)
    return grads


def reference(m, ids, targets, dloss):
    leaf = lambda t: t.double().requires_grad_()      # noqa: E731
    table, w_in, w_out, gates = leaf(m["table"]), [leaf(w) for w in m["w_in"]], [leaf(w) for w in m["w_out"]], [leaf(z) for z in m["gates"]]
    rms = lambda a, w: a / (a.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w      # noqa: E731
    x = table[ids] * 2.0
    for b in range(BLOCKS):
        x = x + SCALE * torch.sigmoid(gates[b]) * rms(block64(m["params"][b], rms(x, w_in[b])), w_out[b])
    z = rms(x, w_in[-1]) @ table.t()
    keep = targets >= 0
    loss = torch.where(keep, torch.logsumexp(z, 1) - z.gather(1, targets.clamp(min=0)[:, None])[:, 0], 0.0)
    (loss * dloss.double()).sum().backward()
    return loss.detach(), {"table": table.grad, "w_in": [w.grad for w in w_in], "w_out": [w.grad for w in w_out], "gates": [z.grad for z in gates]}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_losses_and_gradients_of_a_model(kb, dtype):
    m, ids, targets = model(40, dtype)
    heads = [[kb.VQLayer(p) for p in Ps] for Ps in m["params"]]
    dloss = torch.full((N,), 1.0 / N, device="cuda")
    saved = forward(kb, m, heads, ids, targets)
    grads = backward(kb, m, ids, targets, saved, dloss)
    loss, ref = reference(m, ids, targets, dloss)
    # fp32: KAN heads are within 1e-5 of their largest output, which norms of rows of about that rms pass on; two blocks, and
    # ten for what an output far below the largest makes of it.  bf16: rows and gradients in front of the loss are rounded (2^-9
    # each, rms of 2^-9 / sqrt(3) and smaller), the table's gradient twice.
    tol = 2e-4 if dtype == torch.float32 else 2.0 ** -7
    far = lambda a, b: float((a.double() - b).norm() / b.norm())      # noqa: E731
    assert far(saved[4], loss) <= tol
    for k, want in ref.items():
        for a, b in zip(grads[k] if isinstance(want, list) else [grads[k]], want if isinstance(want, list) else [want]):
            assert far(a, b) <= tol, (k, far(a, b))


def test_one_token_at_a_time(kb):
    """Decoding: a token alone takes the same values as in its batch (KAN heads of one row run other kernels: 1e-5 of the
    largest, which the norm behind passes on), from a captured graph."""
    m, ids, targets = model(50, torch.float32)
    heads = [[kb.VQLayer(p) for p in Ps] for Ps in m["params"]]
    saved = forward(kb, m, heads, ids, targets)
    token, target, gates = ids[:1].clone(), targets[:1].clone(), [z[:1].clone() for z in m["gates"]]
    one = dict(m, gates=gates)
    forward(kb, one, heads, token, target)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            out = forward(kb, one, heads, token, target)
    for n in (3, 77, 0, N - 1):
        token.copy_(ids[n:n + 1])
        target.copy_(targets[n:n + 1])
        for z, all_z in zip(gates, m["gates"]):
            z.copy_(all_z[n:n + 1])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0][0][0], saved[0][0][n])                       # the looked-up row
        assert float((out[3][0] - saved[3][n]).abs().max()) <= 1e-3            # two blocks, 1e-5 of outputs, the norms' gains below 50
        assert abs(float(out[5][0]) - float(saved[5][n])) <= 2e-3
