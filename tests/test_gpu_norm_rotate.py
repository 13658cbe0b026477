"""Norm of queries and keys with the position rotation, and its gradients, against the formulas in 64 bits."""
import pytest
import torch

import cache_reference as ref
import paper_2506_22169_amd as mcf

pytestmark = pytest.mark.gpu

# batch (0: rows without a batch dimension), tokens, heads of q and of k, size, rotated part
SHAPES = [(0, 1, 1, 1, 16, 16), (0, 3, 5, 2, 64, 64), (2, 7, 8, 1, 128, 128), (1, 33, 3, 3, 80, 32), (3, 1, 4, 0, 96, 96), (0, 130, 9, 4, 192, 64),
          (1, 5, 2, 2, 256, 256), (0, 2, 3, 1, 512, 512), (0, 17, 2, 1, 48, 0), (0, 700, 13, 3, 112, 112)]


def _rows(gen, batch, tokens, heads, size, dtype, packed):
    """Rows, or a slice of wider ones (strides of a projection)."""
    lead = (batch, tokens) if batch else (tokens,)
    if packed:
        return torch.randn(*lead, heads, size, generator=gen).to(dtype)
    return torch.randn(*lead, heads + 3, size + 8, generator=gen).to(dtype)[..., 2:2 + heads, :size]


def _place(x, like):
    """A device tensor with the strides of `like`."""
    wide = torch.zeros(like.untyped_storage().nbytes() // 2, dtype=x.dtype, device="cuda").as_strided(like.shape, like.stride(), like.storage_offset())
    wide.copy_(x)
    return wide


def _problem(shape, dtype, norm, interleaved, packed, seed, positions="each"):
    batch, tokens, hq, hk, size, rotary = shape
    gen = torch.Generator().manual_seed(seed)
    q = _rows(gen, batch, tokens, hq, size, dtype, packed)
    k = _rows(gen, batch, tokens, hk, size, dtype, packed) if hk else None
    wq, wk = ((1 + 0.2 * torch.randn(size, generator=gen)).to(dtype) for _ in range(2)) if norm else (None, None)
    cos, sin = ref.tables(rotary, 2 * tokens + 5) if rotary else (None, None)
    lead = (batch, tokens) if batch and positions == "each" else (tokens,)
    at = torch.randint(0, 2 * tokens + 5, lead, generator=gen) if positions else None
    return q, k, cos, sin, at, wq, wk, gen


def _dev(t):
    return None if t is None else t.cuda()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("norm,interleaved,packed", [(True, False, True), (True, True, False), (False, False, False), (False, True, True)])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(shape, norm, interleaved, packed, dtype):
    q, k, cos, sin, at, wq, wk, _ = _problem(shape, dtype, norm, interleaved, packed, 100 + shape[1])
    full = at if at.dim() == q.dim() - 2 else at.expand(q.shape[:-2])
    qo, ko = mcf.norm_rotate(_place(q, q), None if k is None else _place(k, k), _dev(cos), _dev(sin), at.cuda() if packed else at.int().cuda(), _dev(wq), _dev(wk),
                             eps=1e-5, interleaved=interleaved)
    for name, x, w, got in (("q", q, wq, qo), ("k", k, wk, ko)):
        if x is None:
            assert got is None
            continue
        want = ref.norm_rotate(x, cos, sin, full, w, 1e-5, interleaved)
        bound = ref.norm_rotate_bound(x, want, cos, w, 1e-5, interleaved, dtype)
        assert got.shape == x.shape and got.dtype == dtype
        ref.check(got, want, bound, dtype, name)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("norm,interleaved,packed", [(True, False, False), (True, True, True), (False, False, True)])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(shape, norm, interleaved, packed, dtype):
    q, k, cos, sin, at, wq, wk, gen = _problem(shape, dtype, norm, interleaved, packed, 200 + shape[1])
    full = at if at.dim() == q.dim() - 2 else at.expand(q.shape[:-2])
    dq = torch.randn(q.shape, generator=gen).to(dtype)
    dk = None if k is None else torch.randn(k.shape, generator=gen).to(dtype)
    args = (_place(q, q), None if k is None else _place(k, k), _dev(cos), _dev(sin), at.cuda(), _dev(wq), _dev(wk))
    got = mcf.norm_rotate_backward(_dev(dq), _dev(dk), *args, eps=1e-5, interleaved=interleaved)
    again = mcf.norm_rotate_backward(_dev(dq), _dev(dk), *args, eps=1e-5, interleaved=interleaved)
    for name, x, dy, w, dx, dw in (("q", q, dq, wq, got[0], got[2]), ("k", k, dk, wk, got[1], got[3])):
        if x is None:
            assert dx is None and dw is None
            continue
        want, want_w, bx, bw = ref.norm_rotate_backward(dy, x, cos, sin, full, w, 1e-5, interleaved)
        ref.check(dx, want, bx, dtype, "d" + name)
        if w is None:
            assert dw is None
        else:
            assert dw.dtype == torch.float32
            ref.check(dw, want_w, bw, torch.float32, "weight of " + name)
    for a, b in zip(got, again):  # sums in an order that the shapes fix
        assert a is b is None or torch.equal(a, b)


def test_gradients_against_differences():
    """The gradients of a weighted sum of the results, against central differences of the 64-bit form."""
    gen = torch.Generator().manual_seed(7)
    x, dy, w = torch.randn(1, 2, 32, generator=gen), torch.randn(1, 2, 32, generator=gen).half(), (1 + 0.3 * torch.randn(32, generator=gen)).half()
    x = x.half()
    cos, sin = ref.tables(32, 9)
    at = torch.tensor([4])
    dx, _, dw, _ = mcf.norm_rotate_backward(dy.cuda(), None, x.cuda(), None, cos.cuda(), sin.cuda(), at.cuda(), w.cuda(), eps=1e-5)

    def loss(xx, ww):
        return (ref.turn(ref.normed(xx, ww, 1e-5), cos, sin, at, False) * dy.double()).sum().item()

    h = 2.0 ** -12
    for h_i in range(2):
        for e in (0, 5, 16, 31):
            d = torch.zeros(1, 2, 32, dtype=torch.float64)
            d[0, h_i, e] = h
            want = (loss(x.double() + d, w.double()) - loss(x.double() - d, w.double())) / (2 * h)
            # third derivatives are of order 10 here: h^2 of them, and a rounding of the result to fp16
            assert abs(dx[0, h_i, e].item() - want) <= 2.0 ** -11 * abs(want) + 2.0 ** -18
    for e in (0, 5, 16, 31):
        d = torch.zeros(32, dtype=torch.float64)
        d[e] = h
        want = (loss(x.double(), w.double() + d) - loss(x.double(), w.double() - d)) / (2 * h)
        assert abs(dw[e].item() - want) <= 2.0 ** -18 * (1 + abs(want))


def test_in_place_and_float_weights():
    q, k, cos, sin, at, wq, wk, gen = _problem((0, 11, 4, 2, 64, 64), torch.bfloat16, True, False, True, 3)
    want = mcf.norm_rotate(q.cuda(), k.cuda(), cos.cuda(), sin.cuda(), at.cuda(), wq.cuda(), wk.cuda())
    same = mcf.norm_rotate(q.cuda(), k.cuda(), cos.cuda(), sin.cuda(), at.cuda(), wq.float().cuda(), wk.float().cuda())
    qd, kd = q.cuda(), k.cuda()
    out = mcf.norm_rotate(qd, kd, cos.cuda(), sin.cuda(), at.cuda(), wq.cuda(), wk.cuda(), q_out=qd, k_out=kd)
    assert out[0].data_ptr() == qd.data_ptr()
    for a, b, c in zip(want, same, out):
        assert torch.equal(a, b) and torch.equal(a, c)
    # gradients where the gradients were, and results laid out by heads, as the softmax chain takes them
    dq, dk = torch.randn(q.shape, generator=gen).bfloat16().cuda(), torch.randn(k.shape, generator=gen).bfloat16().cuda()
    args = (q.cuda(), k.cuda(), cos.cuda(), sin.cuda(), at.cuda(), wq.cuda(), wk.cuda())
    plain = mcf.norm_rotate_backward(dq, dk, *args)
    moved = mcf.norm_rotate_backward(dq, dk, *args, q_out=dq, k_out=dk)
    assert moved[0].data_ptr() == dq.data_ptr() and all(torch.equal(a, b) for a, b in zip(plain, moved))
    by_head = torch.empty(4, 11, 64, dtype=torch.bfloat16, device="cuda")
    mcf.norm_rotate(q.cuda(), None, cos.cuda(), sin.cuda(), at.cuda(), wq.cuda(), q_out=by_head.transpose(0, 1))
    assert torch.equal(by_head.transpose(0, 1), want[0])


def test_positions():
    """None counts tokens; positions outside of the tables give NaN in the rotated elements, there and nowhere else."""
    q, _, cos, sin, _, _, _, _ = _problem((2, 9, 2, 0, 64, 32), torch.float16, False, False, True, 5)
    plain = mcf.norm_rotate(q.cuda(), None, cos.cuda(), sin.cuda())[0]
    assert torch.equal(plain, mcf.norm_rotate(q.cuda(), None, cos.cuda(), sin.cuda(), torch.arange(9).cuda())[0])
    at = torch.tensor([0, 1, -1, 3, 2 ** 31 - 1, 5, cos.shape[0], cos.shape[0] - 1, -2 ** 31], dtype=torch.int32)
    for p in (at, at.long(), torch.where(at == 2 ** 31 - 1, 2 ** 62, at.long())):
        y = mcf.norm_rotate(q.cuda(), None, cos.cuda(), sin.cuda(), p.cuda())[0].cpu()
        bad = torch.tensor([2, 4, 6, 8])
        assert torch.isnan(y[:, bad, :, :32]).all() and torch.equal(y[:, bad, :, 32:], q[:, bad, :, 32:])
        good = torch.tensor([0, 1, 3, 5, 7])
        assert not torch.isnan(y[:, good]).any()


def test_empty():
    for shape in ((0, 4, 64), (5, 0, 64)):
        q = torch.zeros(shape, dtype=torch.float16, device="cuda")
        assert mcf.norm_rotate(q)[0].shape == shape
        w = torch.ones(64, dtype=torch.float16, device="cuda")
        dx, _, dw, _ = mcf.norm_rotate_backward(q, None, q, q_weight=w)
        assert dx.shape == shape and torch.equal(dw, torch.zeros(64, device="cuda"))


def test_infinities_and_zeros():
    """A row of zeros, rows with infinities and NaN: only their own row is touched by them."""
    q = torch.randn(6, 2, 64).half()
    q[1] = 0
    q[2, 0, 3] = float("inf")
    q[4, 1, 60] = float("nan")
    w = torch.ones(64, dtype=torch.float16)
    y = mcf.norm_rotate(q.cuda(), None, q_weight=w.cuda())[0].cpu()
    want = ref.norm_rotate(q, None, None, None, w, 1e-6, False)
    assert torch.equal(y[1], torch.zeros(2, 64).half())
    assert torch.isnan(y[4, 1]).all() and torch.isnan(y[2, 0, 3]) and (y[2, 0, :3] == 0).all()
    good = torch.tensor([True, True, False, True, False, True])
    ref.check(y[good], want[good], ref.norm_rotate_bound(q[good], want[good], None, w, 1e-6, False, torch.float16), torch.float16)


def test_stream_and_graph():
    q, k, cos, sin, at, wq, wk, gen = _problem((1, 300, 8, 2, 128, 128), torch.bfloat16, True, False, True, 8)
    dq, dk = torch.randn(q.shape, generator=gen).bfloat16().cuda(), torch.randn(k.shape, generator=gen).bfloat16().cuda()
    args = (q.cuda(), k.cuda(), cos.cuda(), sin.cuda(), at.cuda(), wq.cuda(), wk.cuda())
    want = mcf.norm_rotate(*args) + mcf.norm_rotate_backward(dq, dk, *args)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    on_s = mcf.norm_rotate(*args, stream=s)
    s.synchronize()
    assert torch.equal(on_s[0], want[0]) and torch.equal(on_s[1], want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = mcf.norm_rotate(*args) + mcf.norm_rotate_backward(dq, dk, *args)
    for rep in range(4):
        for t in got:
            t.fill_(-3.0)
        junk = [torch.full((1 << i,), float("nan"), device="cuda") for i in range(10, 20)]
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), rep
        del junk
