"""kan_lookup_forward / kan_lookup_backward with scales and rows that are no numbers."""
import pytest

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


@pytest.mark.parametrize("scale", [float("inf"), -float("inf"), float("nan"), 2.0])
@pytest.mark.parametrize("N,D,dtype", [(5, 3, F32), (64, 1000, BF16), (5000, 520, F16)])
def test_an_id_that_names_no_row_gives_zeros_whatever_the_scale(kb, N, D, dtype, scale):
    g = torch.Generator(device="cuda").manual_seed(N)
    table = torch.randn((40, D), generator=g, device="cuda").to(dtype)
    ids = torch.randint(-20, 60, (N,), generator=g, device="cuda")
    none = (ids < 0) | (ids >= 40)
    y = kb.kan_lookup_forward(table, ids, scale=scale)
    assert bool(none.any()) and not y[none].any()
    want = (table[ids[~none]].float() * scale).to(dtype)
    assert torch.equal(y[~none].nan_to_num(nan=7.0), want.nan_to_num(nan=7.0))
    # the gradient of rows that no id names
    dt = kb.kan_lookup_backward(torch.ones((N, D), dtype=dtype, device="cuda"), torch.where(ids < 10, -1, ids), 40, scale=scale)
    assert not dt[:10].any()
