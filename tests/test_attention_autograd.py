"""What the attention binding does where torch differentiates around it:
forward mode, tensors written in place, gradients in unusual memory."""
import pytest

torch = pytest.importorskip("torch")

from torch.autograd import forward_ad  # noqa: E402

import paper_2608_16491_amd as F  # noqa: E402

# the refusals that come before any GPU is touched run on the CPU too
DEVICES = ["cpu", pytest.param("cuda", marks=pytest.mark.gpu)]


def tensors(device, b=2, tq=3, tk=20, h=4, kv=2, d=64, dtype=torch.bfloat16, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(shape, generator=g).to(dtype).to(device) for shape in ((b, tq, h, d), (b, tk, kv, d), (b, tk, kv, d))]


def calls(device):
    """Every operator with its arguments by name, and those that hold real numbers."""
    q, k, v = tensors(device)
    f = dict(device=device, dtype=torch.float32)
    n = dict(device=device, dtype=torch.int32)
    attend = dict(q=q, k=k, v=v, slopes=torch.ones(4, **f), at_q=torch.zeros((2, 3), **f), at_k=torch.zeros((2, 20), **f),
                  weights=torch.zeros((2, 2, 20), **f), weights_out=torch.zeros((2, 2, 20), **f))
    shared = dict(q=q[:, 0].contiguous(), k=k[0], v=v[0], k_pages=k, v_pages=v, slopes=torch.ones(4, **f))
    cache = dict(k=k, v=v, weights=torch.zeros((2, 2, 20), **f))
    return [(F.attend, attend, {}), (F.attend_shared, shared, dict(pages=torch.zeros((2, 1), **n), lengths=torch.ones(2, **n))),
            (F.evict, cache, dict(positions=None, lengths=torch.full((2,), 20, **n), keep=10))]


@pytest.mark.parametrize("device", DEVICES)
@pytest.mark.parametrize("no_grad", [False, True])
def test_tangents_are_refused(device, no_grad):
    for fn, real, others in calls(device):
        for name in real:
            with forward_ad.dual_level(), torch.set_grad_enabled(not no_grad):
                dual = {name: forward_ad.make_dual(real[name], torch.ones_like(real[name]))}
                with pytest.raises(ValueError, match=f"^{name} carries a tangent"):
                    fn(**{**real, **dual}, **others)


@pytest.mark.gpu
def test_calls_within_a_dual_level_whose_tensors_have_no_tangent():
    for fn, real, others in calls("cuda"):
        want = fn(**real, **others)
        with forward_ad.dual_level():
            got = fn(**real, **others)
        assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.gpu
def test_a_tangent_of_the_outputs_gradient_is_refused():
    # forward over reverse, of a factor behind the call
    q, k, v = (t.requires_grad_() for t in tensors("cuda"))
    out = F.attend(q, k, v)
    with forward_ad.dual_level():
        dout = forward_ad.make_dual(torch.ones_like(out), torch.ones_like(out))
        with pytest.raises(ValueError, match="carries a tangent"):
            torch.autograd.grad(out, (q, k, v), dout)


@pytest.mark.gpu
@pytest.mark.parametrize("same", [False, True])
def test_weights_written_in_place_are_seen_by_autograd(same):
    # an earlier product kept the tensor for its gradient: once written, that gradient must not be computed from it
    q, k, v = tensors("cuda")
    w, into = (torch.rand((2, 2, 20), device="cuda") for _ in range(2))
    into = w if same else into
    x = torch.rand((2, 2, 20), device="cuda", requires_grad=True)
    y, before = (x * into).sum(), into._version
    with torch.no_grad():
        F.attend(q, k, v, weights=w, weights_out=into)
    assert into._version > before and (same or w._version == 0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    # a view of a larger tensor, of which autograd counts one version for all
    whole = torch.rand((2, 2, 2, 20), device="cuda")
    y = (x * whole[1]).sum()
    F.attend(q, k, v, weights=w, weights_out=whole[0])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    # tensors without versions are written as before
    with torch.inference_mode():
        kept = torch.zeros((2, 2, 20), device="cuda")
        _, got = F.attend(q, k, v, weights=kept, weights_out=kept)
    assert got is kept and bool(kept.any())
    F.attend(q, k, v, weights=w, weights_out=kept)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradients_handed_in_off_alignment(dtype):
    q, k, v = (t.requires_grad_() for t in tensors("cuda", dtype=dtype))
    out = F.attend(q, k, v)
    g = torch.randn(out.shape, device="cuda").to(dtype)
    want = torch.autograd.grad(out, (q, k, v), g, retain_graph=True)

    def placed(n):
        # contiguous, n values behind a boundary
        t = torch.empty(g.numel() + n, device="cuda", dtype=dtype)[n:].view(g.shape)
        t.copy_(g)
        return t

    wide = torch.empty(*g.shape[:-1], 67, device="cuda", dtype=dtype)       # rows 67 values apart
    wide[..., :64] = g
    for dout in (placed(0), placed(1), placed(3), placed(4), wide[..., :64], g.transpose(1, 2).contiguous().transpose(1, 2)):
        got = torch.autograd.grad(out, (q, k, v), dout, retain_graph=True)
        assert all(torch.equal(a, b) for a, b in zip(want, got)), (dout.data_ptr() % 16, dout.stride())
    # as a program comes by one: an odd number of values joined in front
    want = torch.autograd.grad(F.attend(q, k, v).flatten(), (q, k, v), g.flatten())
    joined = torch.cat([torch.ones(1, device="cuda", dtype=dtype), F.attend(q, k, v).flatten()])
    got = torch.autograd.grad(joined, (q, k, v), torch.cat([torch.ones(1, device="cuda", dtype=dtype), g.flatten()]))
    assert all(torch.equal(a, b) for a, b in zip(want, got))
