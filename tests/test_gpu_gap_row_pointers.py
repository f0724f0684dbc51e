"""Row pointers that decrease or lie out of range: what the calls over gaps of time give for such rows means nothing,
but they write their outputs and their workspace alone."""
import pytest

from .test_gpu_gap_attention import inputs, log, step_inputs
from .test_gpu_sequence import dev

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
GUARD = 4096  # bytes on either side


class Buffer:
    """Memory of a call between guards."""

    def __init__(self, size):
        self.size = size
        self.whole = torch.full((2 * GUARD + size,), 0xA5, dtype=torch.uint8, device="cuda:0")
        self.at = self.whole.data_ptr() + GUARD

    def untouched(self):
        w = self.whole
        return bool((w[:GUARD] == 0xA5).all()) and bool((w[GUARD + self.size:] == 0xA5).all())


def raw(t):
    return t.contiguous().view(torch.uint8).clone()


def pointers(n, few):
    """Row pointers for n tokens, of up to 64 rows or of more."""
    yield [0, 150, 20, -5, 1 << 40, 70, n + 1, -(1 << 62), 1 << 50]
    yield [n + 7, n, 3, 2, 1, 0, n]
    yield [-9, -9, n + 1, n + 1]
    if not few:
        g = torch.Generator().manual_seed(3)
        yield torch.randint(-n, 2 * n, (150,), generator=g).tolist()
        yield [0] + [n + 5, -5] * 60 + [n]


@pytest.mark.parametrize("clear", [0, 1])
@pytest.mark.parametrize("few", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,H,Hk,D", [(200, 2, 1, 32), (333, 4, 4, 50), (130, 2, 2, 128)])
def test_reading_and_gradients(N, H, Hk, D, dtype, few, clear):
    from paper_1108_2580_amd import lib, sequence as s

    q, k, v, bias, bounds, pos, _, do = inputs([N], H, Hk, D, 8, dtype, 91)
    size = q.element_size()
    for ptr in pointers(N, few):
        ptr = ptr if few else (ptr * 70)[:max(len(ptr), 80)]
        log(f"{N} tokens, {H}/{Hk} heads, width {D}, {dtype}, {len(ptr) - 1} rows {ptr[:4]}")
        ptr = dev(torch.tensor(ptr))
        held = (q, k, v, bias, pos, ptr, do)
        before = [raw(t) for t in held]
        dev_, code, shape, hq, hk, hv = s._gaps(q, k, v, bias, bounds, pos, ptr, 0.2)
        shape.clear_unheld = clear
        st, hdo = s._stream(dev_), s._heads(do, "d_out", do.dtype, dev_)
        out, stats, rest = Buffer(N * H * D * size), Buffer(8 * N * H), Buffer(N * H * D * 2)
        need = lib.als_gap_attention_workspace(shape)
        work = Buffer(need)
        rest_at = rest.at if dtype == "bf16" else None
        s._check(lib.als_gap_attention(shape, code, hq, hk, hv, out.at, stats.at, rest_at, work.at if need else None,
                                       need, st))
        outputs = [raw(x.whole) for x in (out, stats, rest)]
        dq, dk, dv, dbias = Buffer(N * H * D * size), Buffer(N * Hk * D * size), Buffer(N * Hk * D * size), Buffer(4 * H * 8)
        need = lib.als_gap_attention_backward_workspace(shape)
        back = Buffer(need)
        s._check(lib.als_gap_attention_backward(shape, code, hdo, hq, hk, hv, out.at, stats.at, rest_at, dq.at, dk.at,
                                                dv.at, dbias.at, back.at, need, st))
        torch.cuda.synchronize()
        for x, name in ((out, "out"), (stats, "stats"), (rest, "rest"), (work, "workspace"), (dq, "dq"), (dk, "dk"),
                        (dv, "dv"), (dbias, "dbias"), (back, "the gradients' workspace")):
            assert x.untouched(), name
        assert dtype == "bf16" or bool((rest.whole == 0xA5).all())
        assert all(torch.equal(raw(x.whole), y) for x, y in zip((out, stats, rest), outputs))
        assert all(torch.equal(raw(t), b) for t, b in zip(held, before))


@pytest.mark.parametrize("few", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,beams,H,Hk,D", [(200, 3, 2, 1, 32), (700, 1, 4, 4, 50), (300, 16, 2, 2, 128)])
def test_steps(N, beams, H, Hk, D, dtype, few):
    from paper_1108_2580_amd import lib, sequence as s

    for ptr in pointers(N, few):
        ptr = ptr if few else (ptr * 70)[:max(len(ptr), 80)]
        lists = len(ptr) - 1
        log(f"{N} tokens, {beams} beams, {H}/{Hk} heads, width {D}, {dtype}, {lists} lists {ptr[:4]}")
        q, _, _, bias, bounds, q_pos, _, _, kp, vp, p_pos, path = step_inputs([1] * lists, beams, 2, H, Hk, D, 8, dtype, 92)
        _, k, v, _, _, pos, _, _ = inputs([N], H, Hk, D, 8, dtype, 93)
        ptr = dev(torch.tensor(ptr))
        held = (q, k, v, bias, q_pos, pos, ptr, kp, vp, p_pos, path)
        before = [raw(t) for t in held]
        dev_, code, shape, hq, hk, hv = s._gaps(q, k, v, bias, bounds, pos, ptr, 0.2)
        heads = [s._Heads(t.data_ptr(), t.stride(1), t.stride(2)) for t in (kp, vp)]
        at = s._GapPath(beams, 2, q_pos.data_ptr(), *heads, kp.stride(0), vp.stride(0), p_pos.data_ptr(), path.data_ptr(), 2)
        out = Buffer(q.numel() * q.element_size())
        need = lib.als_gap_attention_step_workspace(shape, at)
        work = Buffer(need)
        s._check(lib.als_gap_attention_step(shape, at, code, hq, hk, hv, out.at, work.at, need, s._stream(dev_)))
        torch.cuda.synchronize()
        assert out.untouched() and work.untouched()
        assert all(torch.equal(raw(t), b) for t, b in zip(held, before))
