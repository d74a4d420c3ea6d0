"""kan_vocab_loss_forward / kan_vocab_loss_backward at the ends of the sizes and weights that they take, against their definitions
in 64 bits."""
import pytest

from test_gpu_vocab_loss import check_all, draw
from tokens_testlib import HALF, check

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
U = 2.0 ** -24


@pytest.fixture(scope="module")
def kb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2512_15742_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_table_of_all_rows_that_32_bits_count(kb, dtype):
    """2^31 - 1 rows: the last tile ends behind the last number of 32 bits.  All logits but three are one far below 0: a row too many,
    whose logit is 0, would outweigh the others.

    The logits are exact.  lse adds at most V / 32 / 256 statistics of tiles one behind the other, dh a term for every four rows of a
    16th of 2^25 rows and 1,024 pieces; a target's dS is off by its rounding, the others, all equal, by theirs together."""
    V = 2 ** 31 - 1
    table = torch.full((V, 1), -64.0, dtype=dtype, device="cuda")
    special = torch.tensor([0, V // 2, V - 1], device="cuda")
    table[special, 0] = torch.tensor([-60.0, -62.0, -58.0], dtype=dtype, device="cuda")
    h = torch.tensor([[1.0], [0.5]], dtype=dtype, device="cuda")
    t = torch.tensor([V - 1, 0], device="cuda")
    loss, lse = kb.kan_vocab_loss_forward(h, table, t)
    hd, some = h.double(), table[special].double()
    rest = float(V - 3)
    z = hd @ some.t()                                               # [2][3]
    ref = torch.log(z.exp().sum(1) + rest * torch.exp(-64 * hd[:, 0]))
    e = (V / 32 / 256 + 128) * U
    check(lse, ref, torch.full_like(ref, e))
    check(loss, ref - torch.stack([z[0, 2], z[1, 0]]), torch.full_like(ref, e))
    dloss = torch.tensor([1.0, -0.5], device="cuda")
    dh, dt = kb.kan_vocab_loss_backward(h, table, t, lse, dloss)
    p, pr = torch.exp(z - ref[:, None]), torch.exp(-64 * hd[:, 0] - ref)
    hit = torch.zeros_like(p)
    hit[0, 2] = hit[1, 0] = 1.0
    half = HALF[dtype] if dtype != F32 else 2 * U
    w = dloss.double()
    off = half + 4 * e                                              # of an entry of dS
    check(dt[special, 0], (w[:, None] * (p - hit) * hd).sum(0), off * (w.abs()[:, None] * (p + hit) * hd).sum(0))
    size = w.abs() * ((p + hit) @ some[:, 0].abs() + rest * pr * 64)
    check(dh[:, 0], w * ((p - hit) @ some[:, 0] - rest * pr * 64), (off + (2 ** 25 / 16 / 4 + 1024) * U) * size)
    want = float((w * pr * hd[:, 0]).sum())
    limit = off * float((w.abs() * pr * hd[:, 0]).sum()) + HALF[dtype] * abs(want)
    dt[special] = want
    low, high = (float(x) for x in dt.aminmax())
    assert want - limit <= low and high <= want + limit, (low, high, want, limit)


# few tokens over few and many rows, one to many blocks of 32 tokens; columns that end within, with and behind a step of 32; rows and tokens that end within a
# tile of every size; a contraction over the rows in one share and many
FULL_PRECISION = [
    (1, 90001, 33), (3, 40000, 300), (20, 30000, 500), (32, 30011, 257), (33, 70001, 31), (50, 20011, 300), (64, 40003, 96), (65, 30000, 1), (90, 30011, 200),
    (96, 5003, 700), (97, 30011, 95), (128, 30011, 200), (128, 10011, 333), (130, 9000, 1001), (190, 40001, 64), (200, 2000, 1024), (257, 16001, 130),
    (280, 20001, 100), (400, 1300, 260), (400, 30003, 77), (1000, 7001, 190), (1537, 12001, 161), (7, 1003, 1999), (40, 2005, 2101), (128, 5003, 1111),
    (500, 1300, 2000), (1000, 1001, 515),
]


@pytest.mark.parametrize("N,V,D", FULL_PRECISION)
def test_tables_split_in_registers(kb, N, V, D):
    check_all(kb, *draw(N + V + D, N, V, D, F32, ("i64", "i32")[N % 2]), scale=(1.0, 0.5)[D % 2])


@pytest.mark.parametrize("N,V,D", [(40, 20011, 300), (200, 30011, 161)])
def test_full_precision_rows_that_start_anywhere(kb, N, V, D):
    """A table and rows one element behind a boundary of 16 bytes, the table's neighbours no numbers: the same bits as on their own."""
    h, table, t, dloss = draw(3, N, V, D, F32)
    loss, lse = kb.kan_vocab_loss_forward(h, table, t)
    dh, dt = kb.kan_vocab_loss_backward(h, table, t, lse, dloss)

    def between(a):
        whole = torch.full((a.numel() + 33,), float("nan"), device="cuda")
        return whole[17:17 + a.numel()].view(a.shape).copy_(a)
    h2, table2 = between(h), between(table)
    loss2, lse2 = kb.kan_vocab_loss_forward(h2, table2, t)
    dh2, dt2 = kb.kan_vocab_loss_backward(h2, table2, t, lse2, dloss)
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2) and torch.equal(dh, dh2) and torch.equal(dt, dt2)


def test_full_precision_infinite_rows_stay_in_their_tokens(kb):
    """A row of h that is no number spoils its token; the columns behind a table's row belong to the next one and have no part in it."""
    N, V, D = 100, 30011, 75
    h, table, t, dloss = draw(9, N, V, D, F32, left_out=0.0)
    clean = kb.kan_vocab_loss_forward(h, table, t)
    h[3, 7] = float("nan")
    loss, lse = kb.kan_vocab_loss_forward(h, table, t)
    keep = torch.arange(N, device="cuda") != 3
    assert bool(lse[3].isnan()) and torch.equal(loss[keep], clean[0][keep]) and torch.equal(lse[keep], clean[1][keep])
    dl = torch.where(keep, dloss, 0.0)
    dh, _ = kb.kan_vocab_loss_backward(torch.where(keep[:, None], h, 0.0), table, t, clean[1], dl)
    spoiled = table.clone()
    spoiled[V - 1] = float("inf")                   # (no target: its logits are infinite or not numbers in the last row's place alone)
    z_last = kb.kan_vocab_loss_forward(torch.zeros_like(h), table, t)[1]
    assert bool(torch.isfinite(z_last).all()) and bool(torch.isfinite(dh).all())
    lse_bad = kb.kan_vocab_loss_forward(torch.where(keep[:, None], h, 0.0), spoiled, t)[1]
    assert not bool(torch.isfinite(lse_bad[keep]).any())


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("N", [90, 4100])
def test_weights_far_apart(kb, N, dtype):
    """Weights over seven orders of magnitude: an entry of fp16 g is off by 2^-39 of the largest weight beside its own rounding, of the other types by
    its rounding alone (the bounds of Loss.grads)."""
    h, table, t, dloss = draw(33, N, 3001, 64, dtype)
    spread = torch.rand(N, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") * -7
    check_all(kb, h, table, t, dloss.sign() * 10 ** (spread + 1), scale=1.0)
