"""Matrices near the limits of a dimension: sizes that have to be cut into launches, or whose rows pass 31 bits."""
import pytest

pytestmark = pytest.mark.gpu


def _room(gigabytes):
    import torch
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes << 30:
        pytest.skip("needs %d GB of device memory" % gigabytes)


def test_expansion_of_few_very_long_rows():
    # 33 rows of 2^30: more than 2^31 threads' values within the first 128 rows
    import torch
    from paper_1509_04210_b200 import learner as L

    _room(125)
    rows, cols = 33, 1 << 30
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    for r in range(rows):
        x[r].normal_(generator=torch.Generator("cuda").manual_seed(r))
    pick = [0, 31, 32]
    few = x[pick]
    q = L.mx4_quantize(x)
    back = L.mx4_dequantize(q, out=x)
    want = L.mx4_dequantize(L.mx4_quantize(few))
    for i, r in enumerate(pick):
        assert torch.equal(back[r], want[i])
    del x, back, few, want, q
    torch.cuda.empty_cache()


@pytest.mark.parametrize("tokens", [(1 << 31) // 3 + 200_001])
def test_f32_gradients_of_very_many_tokens(tokens):
    # their three planes together have more than 2^31 rows.  A few tokens count, one of them at each end and around the
    # thirds; each needs all three planes (21 bits), and so does their sum, exactly.
    import torch
    from paper_1509_04210_b200 import learner as L

    _room(125)
    saved = L.act8_save(torch.ones((tokens, 1), dtype=torch.bfloat16, device="cuda"))
    dy = torch.zeros((tokens, 1), device="cuda")
    value = 1.0 + 2.0 ** -9 + 2.0 ** -17
    for t in (0, tokens // 3, 2 * tokens // 3, tokens - 1):
        dy[t] = value
    got = L.act8_weight_grad(dy, saved)
    assert float(got) == 4 * value
    assert float(L.act8_weight_grad(dy, saved, torch.bfloat16)) == float(torch.tensor(4 * value).bfloat16())
    L.sync()
    del saved, dy
    torch.cuda.empty_cache()
