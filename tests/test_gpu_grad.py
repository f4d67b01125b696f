"""iabn_grad_norm and iabn_grad_clip on the GPU against their definition in 64 bits."""

from __future__ import annotations

import pytest
import torch

import paper_1712_02616_amd as iabn
import sublayer_oracle as oracle
from gpu_helpers import say

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]

INF, NAN = float("inf"), float("nan")
DTYPES = (torch.float32, torch.float16, torch.bfloat16)
U32 = 2.0 ** -24


def tensors(sizes, seed=1, std=0.5, shift=0):
    """One tensor of each size, the types in turn, `shift` elements off alignment."""
    gen = torch.Generator().manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        flat = torch.zeros(n + shift, dtype=DTYPES[i % 3])
        flat[shift:] = (torch.randn(n, generator=gen) * std).to(DTYPES[i % 3])
        out.append(flat.cuda()[shift:])
    return out


def norm_of(grads):
    return float(torch.stack([g.double().square().sum() for g in grads]).sum().sqrt()) if grads else 0.0


def run(grads, max_norm, in_place=False, stream=None):
    say("grads %d tensors, max_norm %g in_place=%s" % (len(grads), max_norm, in_place))
    want = norm_of(grads)
    norm = torch.full((3,), NAN, device="cuda")
    torch.cuda.synchronize()
    assert iabn.iabn_grad_norm(grads, norm[1:2], stream=stream) is not None
    torch.cuda.synchronize()
    # 64-bit sums, rounded once.
    got = float(norm[1])
    assert abs(got - want) <= want * (U32 + 1e-12) + 2.0 ** -149, (got, want)
    assert torch.isnan(norm[0]) and torch.isnan(norm[2])
    before = [g.clone() for g in grads]
    outs = grads if in_place else [torch.full_like(g, 7.0) for g in grads]
    torch.cuda.synchronize()
    iabn.iabn_grad_clip(grads, outs, norm[1:2], max_norm, stream=stream)
    torch.cuda.synchronize()
    factor = min(1.0, max_norm / (got + 1e-6))
    for i, (b, o) in enumerate(zip(before, outs)):
        if factor == 1.0:
            assert torch.equal(b, o), i
        v = b.cpu().double() * factor  # the factor and the product: a rounding each
        oracle.check("tensor %d" % i, o, v, 2 * U32 * v.abs(), b.dtype)
    return got


@pytest.mark.parametrize("sizes", [(1,), (7,), (8, 9, 4096, 4097), (0, 5, 0), (100000, 3, 2048, 1000003),
                                   tuple(range(1, 300)), (5 << 20, 1, 3 << 20)])
@pytest.mark.parametrize("max_norm", [1e-3, 1e9, 0.0])
def test_lists(sizes, max_norm):
    run(tensors(sizes), max_norm)
    run(tensors(sizes), max_norm, in_place=True)


@pytest.mark.parametrize("shift", [1, 3, 4])
def test_unaligned(shift):
    run(tensors((1000, 77, 40000, 8191), shift=shift), 0.5)


@pytest.mark.parametrize("count", [127, 128, 129, 256, 1000])
def test_more_tensors_than_one_launch_takes(count):
    run(tensors([1 + 37 * i % 5000 for i in range(count)]), 1.0)


def test_no_tensors():
    norm = torch.full((1,), NAN, device="cuda")
    iabn.iabn_grad_norm([], norm)
    assert float(norm) == 0.0
    iabn.iabn_grad_clip([], [], norm, 1.0)
    run(tensors((0, 0, 0)), 1.0)


def test_squares_do_not_overflow():
    g = [torch.full((1000,), 1e25, device="cuda"), torch.full((10,), 1e-30, device="cuda")]
    run(g, 1.0)
    small = [torch.full((1000,), 1e-30, device="cuda")]
    run(small, 1.0)
    zero = [torch.zeros(100, device="cuda")]
    assert run(zero, 1.0) == 0.0
    largest = [torch.full((64,), torch.finfo(torch.float32).max, device="cuda")]
    norm = torch.zeros(1, device="cuda")
    assert float(iabn.iabn_grad_norm(largest, norm)) == INF


def test_nonfinite():
    g = [torch.ones(50, device="cuda"), torch.ones(5000, device="cuda").half()]
    norm = torch.zeros(1, device="cuda")
    g[1][77] = INF
    assert float(iabn.iabn_grad_norm(g, norm)) == INF
    outs = iabn.iabn_grad_clip(g, [torch.empty_like(t) for t in g], norm, 1.0)
    assert (outs[0] == 0).all() and torch.isnan(outs[1][77]) and int(torch.isnan(outs[1]).sum()) == 1
    g[1][77] = NAN
    assert torch.isnan(iabn.iabn_grad_norm(g, norm)).all()
    outs = iabn.iabn_grad_clip(g, [torch.empty_like(t) for t in g], norm, 1.0)
    assert all(torch.isnan(t).all() for t in outs)
    # No limit leaves everything as it is.
    norm.fill_(3.0)
    outs = iabn.iabn_grad_clip(g[:1], [torch.empty_like(g[0])], norm, INF)
    assert torch.equal(outs[0], g[0])


def test_shapes_and_kinds_of_lists():
    """Any shapes, a tuple, a generator, parameters; the same tensor twice counts
    twice."""
    a = torch.randn(3, 5, 7, device="cuda")
    b = torch.nn.Parameter(torch.randn(11, device="cuda"))
    norm = torch.empty((), device="cuda")
    want = norm_of([a, b.detach()])
    for grads in ((a, b.detach()), [a, b], (t for t in (a, b.detach()))):
        got = float(iabn.iabn_grad_norm(grads, norm))
        assert abs(got - want) <= 2 * U32 * want
    assert abs(float(iabn.iabn_grad_norm([a, a], norm)) - norm_of([a, a])) <= 2 * U32 * norm_of([a, a])


def test_another_stream_and_workspace():
    st = torch.cuda.Stream()
    g = tensors((100000, 5000))
    run(g, 0.1, stream=st)
    run(g, 0.1, stream=st.cuda_stream)
    need = iabn.iabn_grad_norm_workspace_size([t.numel() for t in g])
    norms = []
    for fill in (0, 255):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        norms.append(iabn.iabn_grad_norm(g, torch.empty(1, device="cuda"), workspace=ws))
    assert torch.equal(*norms)


def test_a_tensor_past_32_bits():
    n = (1 << 32) + 12345
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[0], g[1 << 31], g[-1] = 3.0, 4.0, 12.0
    norm = torch.empty(1, device="cuda")
    assert float(iabn.iabn_grad_norm([g], norm)) == 13.0
    iabn.iabn_grad_clip([g], [g], norm, 6.5)
    assert [float(g[i]) for i in (0, 1 << 31, n - 1)] == [1.5, 2.0, 6.0]
