"""kan_vocab_loss_forward / kan_vocab_loss_backward at the ends of the sizes and weights that they take, against their definitions
in 64 bits."""
import pytest

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
