"""norm_rotate recorded for autograd: the gradients are norm_rotate_backward's, of everything that asks for one, and nothing is lost silently."""
import pytest
import torch

import cache_reference as ref
import paper_2506_22169_amd as mcf


def _operands(gen, dtype, size=64, heads=(5, 2), lead=(3, 7), device="cuda"):
    qkv = torch.randn(*lead, heads[0] + 2 * heads[1], size, generator=gen).to(dtype).to(device)
    wq, wk = ((1 + 0.2 * torch.randn(size, generator=gen)).to(dtype).to(device) for _ in range(2))
    cos, sin = (t.to(device) for t in ref.tables(size, 40))
    at = torch.randint(0, 40, lead, generator=gen).to(device)
    return qkv, wq, wk, cos, sin, at


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients(interleaved, dtype):
    gen = torch.Generator().manual_seed(71)
    qkv, wq, wk, cos, sin, at = _operands(gen, dtype)
    leaves = [t.clone().requires_grad_() for t in (qkv, wq, wk)]
    q, k = leaves[0][:, :, :5], leaves[0][:, :, 5:7]
    yq, yk = mcf.norm_rotate(q, k, cos, sin, at, *leaves[1:], eps=1e-5, interleaved=interleaved)
    plain = mcf.norm_rotate(qkv[:, :, :5], qkv[:, :, 5:7], cos, sin, at, wq, wk, eps=1e-5, interleaved=interleaved)
    assert torch.equal(yq, plain[0]) and torch.equal(yk, plain[1]) and not plain[0].requires_grad
    dq, dk = torch.randn(yq.shape, generator=gen).to(dtype).cuda(), torch.randn(yk.shape, generator=gen).to(dtype).cuda()
    torch.autograd.backward((yq, yk), (dq, dk))
    want = mcf.norm_rotate_backward(dq, dk, qkv[:, :, :5], qkv[:, :, 5:7], cos, sin, at, wq, wk, eps=1e-5, interleaved=interleaved)
    assert torch.equal(leaves[0].grad[:, :, :5], want[0]) and torch.equal(leaves[0].grad[:, :, 5:7], want[1]) and (leaves[0].grad[:, :, 7:] == 0).all()
    assert torch.equal(leaves[1].grad, want[2].to(dtype)) and torch.equal(leaves[2].grad, want[3].to(dtype))


@pytest.mark.gpu
def test_one_result_and_one_operand():
    """Only one result is used, only one operand asks; the gradient of a sum, which is one number expanded; no k."""
    gen = torch.Generator().manual_seed(72)
    qkv, wq, wk, cos, sin, at = _operands(gen, torch.bfloat16)
    q, k = qkv[:, :, :5], qkv[:, :, 5:7]
    w = wk.float().requires_grad_()
    yq, yk = mcf.norm_rotate(q, k, cos, sin, at, wq.float(), w)
    yk.sum().backward()
    want = mcf.norm_rotate_backward(torch.zeros_like(yq), torch.ones_like(yk), q, k, cos, sin, at, wq.float(), wk.float())
    assert w.grad.dtype == torch.float32 and torch.equal(w.grad, want[3])
    x = q.detach().clone().requires_grad_()
    y, none = mcf.norm_rotate(x, None, cos, sin, at)
    assert none is None
    y.sum().backward()
    assert torch.equal(x.grad, mcf.norm_rotate_backward(torch.ones_like(y), None, q, None, cos, sin, at)[0])
    with torch.no_grad():
        assert not mcf.norm_rotate(x, None, cos, sin, at)[0].requires_grad
        mcf.norm_rotate(x, None, cos, sin, at, q_out=torch.empty_like(x))


@pytest.mark.gpu
def test_training_step():
    """Through the norm, the rotation and a loss of the scores, against the formulas in 64 bits."""
    gen = torch.Generator().manual_seed(73)
    qkv, wq, wk, cos, sin, at = _operands(gen, torch.float16, heads=(3, 3), lead=(1, 33))
    leaves = [t.clone().requires_grad_() for t in (qkv, wq, wk)]
    q, k = mcf.norm_rotate(leaves[0][:, :, :3], leaves[0][:, :, 3:6], cos, sin, at, *leaves[1:])
    g = torch.randn(3, 33, 33, generator=gen).cuda()
    q32, k32 = (t[0].transpose(0, 1).float() for t in (q, k))
    ((q32 @ k32.transpose(1, 2).contiguous()) * g).sum().backward()
    dq, dk = (g @ k32).half().transpose(0, 1)[None], (g.transpose(1, 2).contiguous() @ q32).half().transpose(0, 1)[None]
    for i, (dy, w) in enumerate(((dq, wq), (dk, wk))):
        x = qkv[:, :, 3 * i:3 * i + 3]
        want, want_w, bx, bw = ref.norm_rotate_backward(dy.detach().cpu(), x.cpu(), cos.cpu(), sin.cpu(), at.cpu(), w.cpu(), 1e-6, False)
        # dy is rounded to fp16 from fp32 sums of either order: a step of each of its elements, of which the row's largest bounds what it moves
        ref.check(leaves[0].grad[:, :, 3 * i:3 * i + 3].detach(), want, bx * (1 + ref.half_step(torch.float16) * 2.0 ** 18), torch.float16)
        ref.check(leaves[1 + i].grad.detach(), want_w, bw + 4 * ref.half_step(torch.float16) * 33 * 3 * dy.abs().max().item(), torch.float16)


@pytest.mark.gpu
def test_other_stream():
    """A recorded call on another stream than the current one, on which its gradients run."""
    gen = torch.Generator().manual_seed(76)
    qkv, wq, wk, cos, sin, at = _operands(gen, torch.float16)
    leaves = [t.clone().requires_grad_() for t in (qkv, wq, wk)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    y = mcf.norm_rotate(leaves[0][:, :, :5], leaves[0][:, :, 5:7], cos, sin, at, *leaves[1:], stream=stream)
    torch.cuda.current_stream().wait_stream(stream)
    dy = [torch.randn(t.shape, generator=gen).half().cuda() for t in y]
    torch.autograd.backward(y, dy)
    want = mcf.norm_rotate_backward(*dy, qkv[:, :, :5], qkv[:, :, 5:7], cos, sin, at, wq, wk)
    assert torch.equal(leaves[0].grad[:, :, :7], torch.cat(want[:2], 2))
    assert torch.equal(leaves[1].grad, want[2].half()) and torch.equal(leaves[2].grad, want[3].half())


@pytest.mark.gpu
def test_captures_are_refused():
    """A captured call is refused while the capture goes on, and so are captured gradients of an eager one; the calls themselves are captured."""
    gen = torch.Generator().manual_seed(74)
    qkv, wq, wk, cos, sin, at = _operands(gen, torch.bfloat16)
    q, w = qkv[:, :, :5], wq.clone().requires_grad_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        alive, _ = mcf.norm_rotate(q, None, cos, sin, at, w)  # an eager graph of the same leaf
        dy = torch.ones_like(alive)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        with pytest.raises(mcf.McfError, match="captured") as refused:
            mcf.norm_rotate(q, None, cos, sin, at, w)
        with pytest.raises(mcf.McfError, match="captured"):
            alive.backward(dy)
        with torch.no_grad():
            y, _ = mcf.norm_rotate(q, None, cos, sin, at, w)
            grads = mcf.norm_rotate_backward(dy, None, q, None, cos, sin, at, w)
    assert refused.value.status == 2 and w.grad is None
    want = mcf.norm_rotate_backward(dy, None, q, None, cos, sin, at, wq)
    for _ in range(3):
        grads[2].fill_(-1.0)
        y.fill_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, alive) and torch.equal(grads[2], want[2]) and torch.equal(grads[0], want[0])


def test_refused():
    """Results in tensors of the caller, and tables that ask for a gradient; checked before the device."""
    gen = torch.Generator().manual_seed(75)
    qkv, wq, wk, cos, sin, at = _operands(gen, torch.float16, device="cpu")
    q = qkv[:, :, :5].clone().requires_grad_()
    for kw in (dict(q_out=q), dict(q_out=torch.empty_like(q)), dict(k=qkv[:, :, 5:7], k_out=qkv[:, :, 5:7])):
        with pytest.raises(mcf.McfError, match="not recorded") as e:
            mcf.norm_rotate(q, cos=cos, sin=sin, positions=at, **kw)
        assert e.value.status == 2
    with pytest.raises(mcf.McfError, match="tables") as e:
        mcf.norm_rotate(qkv[:, :, :5], cos=cos.clone().requires_grad_(), sin=sin, positions=at)
    assert e.value.status == 2
    with torch.no_grad(), pytest.raises(mcf.McfError, match="device"):
        mcf.norm_rotate(q, cos=cos, sin=sin, positions=at, q_out=q)
