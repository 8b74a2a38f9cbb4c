"""The norm of many gradients and their clipping on the GPU, against 64 bits.

Sixteen squares in 32 bits are off by at most 9 * 2^-24 of their sum, the rest is in 64; the root takes half of that, its rounding
adds 2^-24: within 6 * 2^-24.  The factor is off by that and one rounding, the product by one more: 8 * 2^-24, and 2^-8 in bf16."""
import numpy as np
import pytest

import block_reference as ref
from test_gpu_learner import _learner, _torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24

LISTS = {"one": [1], "a cluster's": [20000, 513, 1, 30000], "a cluster's last": [256 * 512 - 15], "too many for one": [256 * 512 - 14], "odd": [1, 2, 3, 15, 16, 17, 0, 31, 33, 511, 513, 8191, 8192, 8193, 100003], "empty among": [0, 5, 0], "sixty-five": list(range(1, 66)),
         "two launches": [7 + i % 50 for i in range(1000)], "large": [3_000_001, 96, 1_234_567]}


def _grads(sizes, dtypes, shift, std=1e-3, seed=0):
    """Tensors that start `shift` elements into their buffers, of the dtypes in turn, and what they hold."""
    torch = _torch()
    rng = np.random.default_rng(seed)
    out, held = [], []
    for i, n in enumerate(sizes):
        t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtypes[i % len(dtypes)]]
        buf = torch.full((n + shift + 8,), float("nan"), dtype=t, device="cuda")
        v = buf[shift:shift + n]
        v.copy_(torch.from_numpy((rng.standard_normal(n) * std).astype(np.float32)).cuda())
        out.append(v)
        held.append(v.float().cpu().numpy())
    return out, held


def _check(got, held, want, dtype):
    for g, h, w in zip(got, held, want):
        g = g.detach().float().cpu().numpy().reshape(-1).astype(np.float64)
        assert (np.abs(g - w) <= 8 * U * np.abs(w) * (1 + 2.0 ** -8) + (2.0 ** -8 * np.abs(w) if dtype == "bf16" else 0.0) + 2.0 ** -140).all()


@pytest.mark.parametrize("name", list(LISTS))
@pytest.mark.parametrize("dtypes", [["f32"], ["bf16"], ["f32", "bf16", "bf16"]])
@pytest.mark.parametrize("shift", [0, 3])
def test_norm_and_clipping(name, dtypes, shift):
    torch, L = _torch(), _learner()
    sizes = LISTS[name]
    grads, held = _grads(sizes, dtypes, shift)
    n, _ = ref.clip(held, 1.0)
    norm = L.grad_norm(grads)
    assert norm.shape == () and abs(norm.item() - n) <= 6 * U * n
    assert torch.equal(norm, L.grad_norm(grads))
    most = n / 3
    _, want = ref.clip(held, float(np.float32(most)))
    before = [g.clone() for g in grads]
    for out in ("f32", "bf16"):                               # into one vector, layer after layer
        t = torch.float32 if out == "f32" else torch.bfloat16
        vector = torch.full((sum(sizes) + 20,), 7.0, dtype=t, device="cuda")
        parts = list(vector[5:5 + sum(sizes)].split(sizes))
        got = L.clip_gradients(grads, most, out=parts)
        assert torch.equal(got, norm) and all(torch.equal(a, b) for a, b in zip(grads, before))
        _check(parts, held, want, out)
        assert (vector[:5] == 7).all() and (vector[5 + sum(sizes):] == 7).all()
    for where in (most, n * 2):                               # in place; nothing to do the second time
        mine = [torch.full((g.numel() + 13,), 7.0, dtype=g.dtype, device="cuda") for g in grads]
        views = [m[5:5 + g.numel()] for m, g in zip(mine, grads)]
        for v, g in zip(views, grads):
            v.copy_(g)
        assert abs(L.clip_gradients(views, where).item() - n) <= 6 * U * n
        if where > n:
            assert all(torch.equal(v, g) for v, g in zip(views, grads))
        else:
            for v, h, w in zip(views, held, want):
                _check([v], [h], [w], "bf16" if v.dtype == torch.bfloat16 else "f32")
        assert all((m[:5] == 7).all() and (m[5 + g.numel():] == 7).all() for m, g in zip(mine, grads))


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-22, 1e22, 1e30, 1e36])
def test_squares_that_a_float_does_not_hold(scale):
    torch, L = _torch(), _learner()
    grads, held = _grads([1000, 77], ["f32"], 1, std=scale / 4)
    n, want = ref.clip(held, scale)
    assert abs(L.grad_norm(grads).item() - n) <= 6 * U * n + 2.0 ** -149
    L.clip_gradients(grads, scale)
    _check(grads, held, want, "f32")


def test_some_large_among_small_ones_and_zeros():
    torch, L = _torch(), _learner()
    g = torch.zeros(50000, device="cuda")
    assert L.grad_norm([g]).item() == 0.0
    L.clip_gradients([g], 0.0)
    assert (g == 0).all()
    g[::1000] = 1e-25
    g[77] = 3.0
    assert L.grad_norm([g]).item() == 3.0
    g[78] = 4e30
    assert L.grad_norm([g]).item() == np.float32(4e30)


def test_norms_that_are_no_numbers():
    torch, L = _torch(), _learner()
    for bad in (float("inf"), -float("inf"), float("nan")):
        g = [torch.ones(5000, device="cuda"), torch.ones(40, device="cuda", dtype=torch.bfloat16)]
        g[0][4321] = bad
        norm = L.clip_gradients(g, 1.0)
        if np.isnan(bad):
            assert torch.isnan(norm) and torch.isnan(g[0]).all() and torch.isnan(g[1]).all()
        else:
            assert torch.isinf(norm) and torch.isnan(g[0][4321]) and torch.isnan(g[0]).sum() == 1 and (g[0].nan_to_num() == 0).all() and (g[1] == 0).all()
    g = [torch.full((100,), 2.0, device="cuda")]
    L.clip_gradients(g, 0.0)
    assert (g[0] == 0).all()
    g = [torch.full((100,), 2.0, device="cuda")]
    L.clip_gradients(g, float("inf"))
    assert (g[0] == 2).all()
    # a norm that is known already
    total = torch.full((1,), 8.0, device="cuda")
    assert L.clip_gradients(g, 4.0, norm=total) is total and (g[0] == 1).all()


def test_shapes_orders_and_refusals():
    torch, L = _torch(), _learner()
    from paper_1509_04210_b200 import binding as rb
    a, b = torch.randn(3, 5, 7, device="cuda"), torch.randn(11, device="cuda")
    n = (a.double().pow(2).sum() + b.double().pow(2).sum()).sqrt().item()
    assert abs(L.grad_norm((a, b)).item() - n) <= 6 * U * n and abs(L.grad_norm([b, a, a[1]]).item() - np.sqrt(n * n + a[1].double().pow(2).sum().item())) <= 8 * U * n
    pool = torch.randn(100, device="cuda")
    kept = pool.clone()
    for call in (lambda: L.grad_norm([]), lambda: L.grad_norm([a.cpu()]), lambda: L.grad_norm([a.half()]), lambda: L.grad_norm([a.transpose(0, 1)]), lambda: L.grad_norm(a.sum()),
                 lambda: L.grad_norm([a.clone().requires_grad_()]), lambda: L.grad_norm([a, None]), lambda: L.grad_norm([a], out=torch.zeros(2, device="cuda")),
                 lambda: L.clip_gradients([a], 1.0, out=[b]), lambda: L.clip_gradients([a], 1.0, out=[a, b]), lambda: L.clip_gradients([a], 1.0, norm=torch.zeros((), device="cuda", dtype=torch.float64))):
        with pytest.raises((ValueError, TypeError)):
            call()
    for grads, out in (([pool, pool], None), ([pool[:50], pool[49:]], None), ([pool[:50], b], [pool[1:51], b]), ([pool[:50]], [pool[1:51]]),
                       ([pool[:50], pool[50:]], [pool[50:], pool[:50]]), ([pool[:50]], [pool[:25].view(torch.bfloat16)]), ([a[0].reshape(-1)[:30], b], [pool[:30], pool[29:40]])):
        with pytest.raises(rb.RudraError, match="overlap"):
            L.clip_gradients(grads, 1e-9, out=out)
    with pytest.raises(rb.RudraError, match="max_norm"):
        L.clip_gradients([pool], -1.0)
    with pytest.raises(rb.RudraError, match="max_norm"):
        L.clip_gradients([pool], float("nan"))
    torch.cuda.synchronize()
    assert torch.equal(pool, kept)
    two = torch.zeros(200, device="cuda")
    L.clip_gradients([pool, pool], 1e-3, out=[two[:100], two[100:]])       # the same gradient twice, read only
    assert torch.equal(two[:100], two[100:]) and abs(two.double().norm().item() - 1e-3) < 1e-8


def test_a_generators_tensors_live_until_the_launch():
    torch, L = _torch(), _learner()

    class Last(torch.Tensor):
        def __del__(self):
            self.plain.fill_(float("nan"))      # on the stream: before the launch it would be the norm's

    def last(g):
        plain = g.float()
        t = plain.as_subclass(Last)
        t.plain = plain
        return t
    grads, held = _grads([700, 3, 40000], ["bf16"], 0)
    n, _ = ref.clip(held, 1.0)
    assert abs(L.grad_norm(last(g) for g in grads).item() - n) <= 6 * U * n
    out = [torch.empty(g.numel(), device="cuda") for g in grads]
    most = float(np.float32(n / 3))
    assert abs(L.clip_gradients((last(g) for g in grads), most, out=(o for o in out)).item() - n) <= 6 * U * n
    _check(out, held, ref.clip(held, most)[1], "f32")
