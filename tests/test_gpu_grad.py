"""Norm and clipping of many gradients against a 64-bit evaluation."""
import pytest
import torch

from paper_2110_15362_b200 import binding as B
from tests.block_util import DT, HALF, TINY, Buffer, gen, normal, within

pytestmark = pytest.mark.gpu
KINDS = ["f32", "f16", "bf16", "f64"]
TILE = {"f32": 8192, "f16": 16384, "bf16": 16384, "f64": 4096}
# squares of a vector summed in binary32: at most 8 roundings of 2^-24, halved by the root; the rounding of the norm
NORM = 5 * 2.0 ** -24


def make(kind, sizes, seed=0, std=1e-2):
    g = gen(seed)
    return [normal(g, (n,), kind, std * 10.0 ** (k % 5 - 2)) for k, n in enumerate(sizes)]


def reference(grads, max_norm):
    norm = torch.stack([(g.double() ** 2).sum() for g in grads]).sum().sqrt()
    return norm, min(1.0, max_norm / (float(norm) + 1e-6))


def clip(grads, max_norm, in_place=False):
    outs = [g if in_place else Buffer(g.shape, g.dtype) for g in grads]
    norm = torch.full((1,), -1.0, dtype=torch.float32, device="cuda")
    ws = B.new_grad_workspace([g.numel() for g in grads])
    ws.fill_(0xFF)
    B.bt_grad_clip_batch(B.grad_items(grads, None if in_place else [b.t for b in outs]), grads[0].dtype, max_norm, norm, ws)
    torch.cuda.synchronize()
    assert in_place or all(b.intact() for b in outs)
    return norm, outs if in_place else [b.t for b in outs]


def check(kind, grads, max_norm, got):
    norm, c = reference(grads, max_norm)
    assert abs(float(got[0]) - float(norm)) <= NORM * float(norm)
    for a, g in zip(got[1], grads):
        want = g.double() * c
        # the factor's error: the norm's and its own rounding; the product's
        within("y", a, want, want.abs() * (HALF[kind] + (2 * NORM + 2.0 ** -23 if kind != "f64" else 1e-14)) + TINY[kind])


def sizes_of(kind):
    t = TILE[kind]
    return [1, 7, 8, t - 1, t, t + 1, 3 * t + 5, 0, 40 * t + 3, 2]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("max_norm", [0.5, 1e6, 0.0, float("inf")])
def test_clip(kind, max_norm):
    grads = make(kind, sizes_of(kind))
    check(kind, grads, max_norm, clip(grads, max_norm))
    copies = [g.clone() for g in grads]
    norm, outs = clip(copies, max_norm, in_place=True)
    check(kind, grads, max_norm, (norm, outs))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("count", [1, 64, 65, 256, 257, 1024, 1025, 2500])
def test_many_tensors(kind, count):
    """Beyond 64, 256 and 1024 tensors: other parameters, several launches."""
    grads = make(kind, [(37 * k) % 1000 + (TILE[kind] if k % 100 == 0 else 0) for k in range(count)], seed=count)
    check(kind, grads, 0.25, clip(grads, 0.25))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_more_tiles_than_ctas(kind):
    grads = make(kind, [TILE[kind] * 900 + 11, TILE[kind] * 300, 5], seed=3)
    check(kind, grads, 0.1, clip(grads, 0.1))


@pytest.mark.parametrize("kind,size", [("f32", 1e30), ("f32", 1e-30), ("bf16", 1e30), ("bf16", 1e-30), ("f32", 1e-22), ("f64", 1e100)])
def test_gradients_of_any_magnitude(kind, size):
    """Squares that overflow or underflow in binary32."""
    grads = [(normal(gen(5), (1000,), "f64") * size).to(DT[kind]), torch.zeros(100, dtype=DT[kind], device="cuda")]
    norm, c = reference(grads, 1.0)
    got, outs = clip(grads, 1.0)
    if size < 1e37:
        assert abs(float(got) - float(norm)) <= NORM * float(norm)
    want = grads[0].double() * c
    within("y", outs[0], want, want.abs() * (HALF[kind] + 2 * NORM + 2.0 ** -23) + 2.0 ** -126)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_infinities_and_nans(kind):
    grads = make(kind, [1000, 9, 40000])
    grads[1][3] = float("inf")
    norm, outs = clip(grads, 1.0)
    assert torch.isinf(norm).all() and torch.isnan(outs[1][3])                   # 0 * inf
    assert not outs[0].any() and not outs[2].any()
    grads[1][3] = float("nan")
    norm, outs = clip(grads, 1.0)
    assert torch.isnan(norm).all() and all(torch.isnan(o).all() for o in outs)


def test_nothing():
    for grads in ([], [torch.empty(0, device="cuda")]):
        norm = torch.full((1,), -1.0, device="cuda")
        B.bt_grad_clip_batch(B.grad_items(grads), torch.float32, 1.0, norm, B.new_grad_workspace([g.numel() for g in grads]))
        assert float(norm) == 0.0


def test_gradients_of_several_types():
    """Sum over the types, then the products of each: what one call gives for all of them as doubles."""
    groups = {k: make(k, [5000, 33, 100000], seed=i) for i, k in enumerate(["f32", "bf16", "f16"])}
    sumsq = torch.full((1,), float("nan"), dtype=torch.float64, device="cuda")
    norm = torch.empty(1, device="cuda")
    want = torch.stack([(g.double() ** 2).sum() for gs in groups.values() for g in gs]).sum()
    for i, (k, gs) in enumerate(groups.items()):
        B.bt_grad_norm_batch(B.grad_items(gs), DT[k], sumsq, norm, B.new_grad_workspace([g.numel() for g in gs]), accumulate=i > 0)
    assert abs(float(sumsq) - float(want)) <= 2 * NORM * float(want) and abs(float(norm) - float(want) ** 0.5) <= NORM * float(want) ** 0.5
    c = min(1.0, 0.3 / (float(want) ** 0.5 + 1e-6))
    for k, gs in groups.items():
        outs = [torch.empty_like(g) for g in gs]
        B.bt_grad_scale_batch(B.grad_items(gs, outs), DT[k], 0.3, sumsq)
        for g, o in zip(gs, outs):
            within(k, o, g.double() * c, (g.double() * c).abs() * (HALF[k] + 2 * NORM + 2.0 ** -23) + TINY[k])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_streams_graphs_and_repeats(kind):
    grads = make(kind, sizes_of(kind), seed=9)
    want_norm, want = clip(grads, 0.5)
    outs, norm = [torch.empty_like(g) for g in grads], torch.empty(1, device="cuda")
    ws = B.new_grad_workspace([g.numel() for g in grads])

    def check_and_clear():
        torch.cuda.synchronize()
        assert torch.equal(norm, want_norm) and all(torch.equal(a, b) for a, b in zip(outs, want))
        for o in outs:
            o.zero_()
        norm.zero_()
        torch.cuda.synchronize()

    items = B.grad_items(grads, outs)
    B.bt_grad_clip_batch(items, DT[kind], 0.5, norm, ws, stream=torch.cuda.Stream())
    check_and_clear()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            B.bt_grad_clip_batch(items, DT[kind], 0.5, norm, ws)
    for _ in range(3):
        for g in graphs:
            g.replay()
        check_and_clear()
