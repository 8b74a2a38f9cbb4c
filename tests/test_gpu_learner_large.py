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
