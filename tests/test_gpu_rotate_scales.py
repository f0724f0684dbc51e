"""Norm and rotation's gradients for rows far from unit scale, whose cubes leave fp32's range. Bounds as in
test_gpu_sequence."""
import pytest

from .test_gpu_sequence import DTYPES, E, U, dev, log, rotate_reference, within

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nb,D", [(False, 64), (True, 37)])
@pytest.mark.parametrize("scale,eps", [(1e13, 1e-6), (1e15, 1e-6), (1e17, 1e-6), (1e-10, 0.0), (1e-14, 0.0),
                                       (1e-16, 0.0), (1e-14, 1e-6)])
def test_gradients_at_any_scale(scale, eps, nb, D, dtype):
    import paper_1108_2580_amd as p

    N, H, dt = 20, 3, DTYPES[dtype]
    g = torch.Generator().manual_seed(D)
    q, k = (dev((torch.randn(N, H, D, generator=g) * scale).to(dt)) for _ in range(2))
    wq, wk = (dev(1 + 0.2 * torch.randn(D, generator=g)) for _ in range(2))
    cos, sin = p.rotary_tables(30, 2 * (D // 4))
    pos = dev(torch.randint(0, 30, (N,), generator=g, dtype=torch.int32))
    args = (q, k, wq, wk, cos, sin, pos, eps, nb)
    dq, dk = (dev(torch.randn(t.shape, generator=g).to(dt)) for t in (q, k))
    log(f"scale {scale}, eps {eps}, neighbours {nb}, width {D}, {dtype}")
    outs = p.norm_rotate(*args)
    grads = p.norm_rotate_backward(dq, dk, *args)
    for i, (x, w, dy, name) in enumerate(((q, wq, dq, "q"), (k, wk, dk, "k"))):
        want, size = rotate_reference(x, w, cos, sin, pos, eps, nb)
        within(outs[i], want, (U if dt == torch.bfloat16 else E) * want.abs() + (D + 12) * E * size + 1e-30, name)
        want, size, want_w, size_w = rotate_reference(x, w, cos, sin, pos, eps, nb, dy)
        within(grads[i], want, (U if dt == torch.bfloat16 else E) * want.abs() + (2 * D + 24) * E * size + 1e-30,
               "d" + name)
        within(grads[2 + i], want_w, (N * H + D + 24) * E * size_w + 1e-30, "d" + name + " weight")
