"""The operators on tensors whose element offsets pass 2^31: rows far apart in one large buffer, a table of more than
2^31 elements.  The same numbers laid out densely give the same bits, since nothing but addresses differs."""
import pytest
import torch

from paper_2502_12996_b200 import ops

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def _device():
    torch.cuda.set_device(0)
    yield
    torch.cuda.empty_cache()


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def far(rows, width, dtype=BF16):
    """[rows, width] with rows 2^27 elements apart: 20 of them pass 2^31."""
    return torch.empty(rows << 27, dtype=dtype, device=DEV).view(rows, 1 << 27)[:, :width]


def test_attention_rows_far_apart():
    T, H, K, D = 20, 2, 1, 64
    wide = far(T, (4 * H + 4 * K) * D)
    assert (T - 1) * wide.stride(0) > 2 ** 31
    g = gen(1)
    cut, at = torch.tensor([0, 3, T], dtype=torch.int32, device=DEV), 0
    t = {}
    for name, heads in (("q", H), ("k", K), ("v", K), ("dout", H), ("out", H), ("dq", H), ("dk", K), ("dv", K)):
        t[name] = wide[:, at:at + heads * D].unflatten(1, (heads, D))
        at += heads * D
    dense = {n: torch.randn((T, t[n].shape[1], D), generator=g, device=DEV).to(BF16) for n in ("q", "k", "v", "dout")}
    for n, v in dense.items():
        t[n].copy_(v)
    out, lse = ops.attention_forward(dense["q"], dense["k"], dense["v"], cut)
    grads = ops.attention_backward(dense["dout"], dense["q"], dense["k"], dense["v"], out, lse, cut)
    _, lse2 = ops.attention_forward(t["q"], t["k"], t["v"], cut, out=t["out"])
    ops.attention_backward(t["dout"], t["q"], t["k"], t["v"], t["out"], lse2, cut, dq=t["dq"], dk=t["dk"], dv=t["dv"])
    assert torch.equal(lse, lse2) and torch.equal(out, t["out"])
    for a, n in zip(grads, ("dq", "dk", "dv")):
        assert torch.equal(a, t[n]), n
    ops.check_device_status()


def test_layer_norm_rows_far_apart():
    T, G, d = 20, 3, 64
    wide = far(T, 3 * G * d)
    x, dy, dx = (wide[:, i * G * d:(i + 1) * G * d].unflatten(1, (G, d))[None] for i in range(3))
    g = gen(2)
    xs, dys, w = (torch.randn(s, generator=g, device=DEV) for s in ((1, T, G, d), (1, T, G, d), (1, d)))
    xs, dys = xs.to(BF16), dys.to(BF16)
    x.copy_(xs), dy.copy_(dys)
    y, mean, rstd = ops.layer_norm_forward(xs, w)
    y2, mean2, rstd2 = ops.layer_norm_forward(x, w)
    assert torch.equal(y, y2) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)
    dw, dw2 = torch.empty_like(w), torch.empty_like(w)
    want = ops.layer_norm_backward(dys, xs, w, mean, rstd, dw)
    ops.layer_norm_backward(dy, x, w, mean, rstd, dw2, dx=dx)
    assert torch.equal(want, dx) and torch.equal(dw, dw2)


def test_loss_rows_far_apart():
    N, V = 20, 1003
    logits = far(N, V)
    g = gen(3)
    x = torch.randn((N, V), generator=g, device=DEV).to(BF16)
    logits.copy_(x)
    ids = torch.randint(0, V, (N, 5), generator=g, device=DEV, dtype=torch.int32)
    t = torch.randn((N, 5), generator=g, device=DEV)
    want = ops.distill_loss(x, ids, t, grad=True)
    got = ops.distill_loss(logits, ids, t, dlogits=logits)
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_embedding_large_table():
    V, d = 1 << 20, 2056                                     # 2.16e9 elements
    table = torch.zeros((1, V, d), dtype=BF16, device=DEV)
    ids = torch.tensor([[V - 1, 0, V - 2, V // 2, V - 1]], dtype=torch.int64, device=DEV)
    rows = torch.randn((5, d), generator=gen(4), device=DEV).to(BF16)
    table[0, ids[0]] = rows
    table[0, V - 1] = rows[4]
    out = ops.embedding_forward(ids, table)
    assert torch.equal(out[0, 1:], rows[1:]) and torch.equal(out[0, 0], rows[4])
    table.fill_(1.0)
    ops.embedding_backward(ids, rows[None], table)
    assert torch.equal(table[0, V - 1], (rows[0].float() + rows[4].float()).to(BF16))
    for i in (1, 2, 3):
        assert torch.equal(table[0, ids[0, i]], rows[i])
    assert int((table != 0).any(-1).sum()) == 4
    far_rows = far(20, d)[None]                               # and rows of the activations far apart
    ids = torch.arange(20, device=DEV, dtype=torch.int32)[None] % 7
    small = torch.randn((1, 7, d), generator=gen(5), device=DEV).to(BF16)
    ops.embedding_forward(ids, small, out=far_rows)
    assert torch.equal(far_rows, small[:, ids[0].long()])
    a, b = torch.empty((1, 7, d), device=DEV), torch.empty((1, 7, d), device=DEV)
    ops.embedding_backward(ids, far_rows, a)
    ops.embedding_backward(ids, far_rows.contiguous(), b)
    assert torch.equal(a, b)
