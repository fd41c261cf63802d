"""The global gradient norm and clipping against 64 bits.  The squares are
summed in 64 bits, so the norm is off by its one rounding to float (2^-24 of
it) and, from the partial sums, by less than another; an output by the
factor's rounding, the product's and, in bf16, half a step (2^-8)."""
import numpy as np
import pytest

from paper_2608_02032_amd import dart

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}


def tdtype(d):
    import torch
    return torch.bfloat16 if d == "bf16" else torch.float32


def tensor(a, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32).reshape(np.shape(a))).to(tdtype(dtype)).cuda()


def f64(t):
    return t.detach().double().cpu().numpy()


def check(grads, before, norm, max_norm, scale, out):
    total = abs(scale) * np.sqrt(sum((b ** 2).sum() for b in before))
    assert norm.shape == () and abs(float(norm) - total) <= 2 * U * total
    if max_norm is None:
        return
    f = scale * min(1.0, max_norm / (total + 1e-6))
    for k, (b, o) in enumerate(zip(before, out)):
        step = 2.0 ** -8 if o.dtype == tdtype("bf16") else 0.0
        ref = b * f
        assert (np.abs(f64(o) - ref) <= (step + 4 * U) * np.abs(ref) + 1e-40).all(), "tensor %d" % k


SHAPES = {
    "one": [(1,)],
    "few": [(3, 5), (7,), (0, 4), (1024, 33), (), (8192,), (8193,), (16385,)],
    "edges": [(n,) for n in (1, 2, 3, 4, 5, 7, 8, 9, 255, 256, 257, 2047, 2048, 2049, 8191, 8192, 8193, 65535, 65537)],
    "many": [(k % 300 + 1,) for k in range(300)] + [(70000,)],
    "table": [(5,)] * 119 + [(3,)],
    "table+1": [(5,)] * 120 + [(3,)],
    "thousand": [(17, 3)] * 1000,
    "large": [(3000, 4001), (2_000_003,)],
    "empty": [(0,), (4, 0)],
    "none": [],
}


@pytest.mark.parametrize("shapes", list(SHAPES))
@pytest.mark.parametrize("dtype,to", [("fp32", ""), ("bf16", ""), ("mixed", ""), ("bf16", "fp32"), ("fp32", "bf16"), ("mixed", "mixed")])
def test_norm_and_clipping(shapes, dtype, to):
    import torch
    rng = np.random.default_rng(len(shapes))
    pick = lambda d, k: d if d != "mixed" else ("fp32", "bf16")[k % 3 == 1]  # noqa: E731
    for max_norm_of, scale in ((0.5, 1.0), (2.0, 1.0), (0.25, 0.125), (3.0, -2.0), (None, 0.5), (np.inf, 0.5), (0.0, 1.0)):
        print("\n[gpu-case] clip %s %s->%s max=%s scale=%s" % (shapes, dtype, to, max_norm_of, scale), flush=True)
        grads = [tensor(rng.standard_normal(s) * 0.01, pick(dtype, k)) for k, s in enumerate(SHAPES[shapes])]
        before = [f64(g) for g in grads]
        total = abs(scale) * np.sqrt(sum((b ** 2).sum() for b in before))
        if max_norm_of is None:
            check(grads, before, dart.grad_norm(grads, scale=scale), None, scale, None)
            assert all(np.array_equal(f64(g), b) for g, b in zip(grads, before))
            continue
        limit = float(np.float32(max_norm_of * total)) if total else max_norm_of
        out = [torch.full(s, 7.0, dtype=tdtype(pick("mixed" if to == "mixed" else to, k + 1)), device="cuda")
               for k, s in enumerate(SHAPES[shapes])] if to else None
        norm = dart.clip_grad_norm(grads, limit, scale=scale, out=out)
        check(grads, before, norm, limit, scale, grads if out is None else out)
        if out is not None:
            assert all(np.array_equal(f64(g), b) for g, b in zip(grads, before))


def test_misaligned_views_of_one_buffer():
    """Gradients that follow each other without gaps; the elements around them stay as they were."""
    import torch
    rng = np.random.default_rng(0)
    sizes = [1, 3, 8, 13, 1024, 8191, 9000, 20001, 5]
    for dtype in ("fp32", "bf16"):
        for to in ("", "fp32", "bf16"):
            print("\n[gpu-case] clip misaligned %s -> %s" % (dtype, to), flush=True)
            buf = tensor(rng.standard_normal(sum(sizes) + 9), dtype)
            obuf = torch.full((sum(sizes) + 16,), 7.0, dtype=tdtype(to or dtype), device="cuda")
            grads, outs, at = [], [], 3
            for n in sizes:
                grads.append(buf[at:at + n])
                outs.append(obuf[at + 2:at + 2 + n])
                at += n
            keep, before = buf.clone(), [f64(g) for g in grads]
            norm = dart.clip_grad_norm(grads, 1.0, out=outs if to else None)
            check(grads, before, norm, 1.0, 1.0, outs if to else grads)
            assert buf[:3].equal(keep[:3]) and buf[at:].equal(keep[at:])
            if to:
                assert buf.equal(keep) and bool((obuf[:5] == 7.0).all()) and bool((obuf[at + 2:] == 7.0).all())


def test_dense_orders_and_refusals():
    import torch
    rng = np.random.default_rng(1)
    a = tensor(rng.standard_normal((40, 30)), "fp32")
    g = [a.t(), tensor(rng.standard_normal((4, 6, 8)), "bf16").permute(2, 0, 1)]
    before = [f64(t) for t in g]
    norm = dart.clip_grad_norm(g, 1.0)
    check(g, before, norm, 1.0, 1.0, g)
    with pytest.raises(ValueError):
        dart.clip_grad_norm([a[:, :10]], 1.0)
    with pytest.raises(ValueError):
        dart.clip_grad_norm([a.t()], 1.0, out=[torch.empty(30, 40, device="cuda")])
    with pytest.raises(ValueError):
        dart.clip_grad_norm([a], 1.0, out=[])
    with pytest.raises(dart.DartError):
        dart.clip_grad_norm([a, a], 1.0)
    with pytest.raises(dart.DartError):
        dart.clip_grad_norm([a, a[3:5]], 1.0)
    with pytest.raises(TypeError):
        dart.clip_grad_norm([a.half()], 1.0)
    with pytest.raises(dart.DartError):
        dart.clip_grad_norm([a], -1.0)
    # reading the same tensor twice is a norm like any other
    want = np.sqrt(2 * (f64(a) ** 2).sum())
    assert abs(float(dart.grad_norm([a, a])) - want) <= 2 * U * want
    assert abs(float(dart.grad_norm(t for t in [a, a])) - want) <= 2 * U * want


def test_extreme_values():
    """Squares past float's range on either side, and what is not finite."""
    import torch
    big = torch.full((1000,), 1e30, device="cuda")
    assert abs(float(dart.grad_norm([big])) / (1e30 * np.sqrt(1000.0)) - 1) <= 1e-6
    small = torch.full((1000,), 1e-30, device="cuda")
    assert abs(float(dart.grad_norm([small])) / (1e-30 * np.sqrt(1000.0)) - 1) <= 1e-6
    g = [torch.ones(5000, device="cuda"), torch.ones(10, device="cuda")]
    g[1][3] = float("nan")
    n = dart.clip_grad_norm(g, 1.0)
    assert bool(torch.isnan(n)) and all(bool(torch.isnan(t).all()) for t in g)
    g = [torch.ones(5000, device="cuda"), torch.ones(10, device="cuda")]
    g[1][3] = float("-inf")
    n = dart.clip_grad_norm(g, 1.0)
    assert float(n) == float("inf") and not bool(g[0].any()) and bool(torch.isnan(g[1][3])) and not bool(g[1][:3].any())


def test_offsets_past_32_bits():
    import torch
    n = (1 << 31) + 1000
    print("\n[gpu-case] clip of %d bf16 elements" % n, flush=True)
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-7:] = 2.0
    g[5] = 3.0
    want = np.sqrt(7 * 4.0 + 9.0)
    norm = dart.clip_grad_norm([g], 1.0)
    assert abs(float(norm) - want) <= 2 * U * want
    assert np.abs(f64(g[-7:]) - 2 / want).max() <= 2.0 ** -8 * 2 / want and not bool(g[6:-7].any())


def test_within_the_limit_nothing_is_written_and_streams():
    import torch
    rng = np.random.default_rng(9)
    g = [tensor(rng.standard_normal(100003), "fp32"), tensor(rng.standard_normal((64, 65)), "bf16")]
    keep = [t.clone() for t in g]
    ref = dart.clip_grad_norm(g, 1e6)
    assert all(a.equal(b) for a, b in zip(g, keep))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):
        norm = dart.grad_norm(g, stream=side)
        junk = [torch.full((1 << 14,), 3.0, device="cuda") for _ in range(8)]
    side.synchronize()
    assert norm.equal(ref) and junk


@pytest.mark.parametrize("to", ["", "fp32", "bf16"])
def test_an_infinite_limit_scales_whatever_the_norm(to):
    """An infinity among the gradients, without a limit: the others are scaled, not lost; a NaN still spoils all."""
    import torch
    for dtype in ("fp32", "bf16"):
        g = [tensor(np.arange(5000) % 7, dtype), tensor(np.ones(10), "fp32")]
        g[1][3] = float("inf")
        before = [f64(t) for t in g]
        out = [torch.full(t.shape, 7.0, dtype=tdtype(to), device="cuda") for t in g] if to else None
        n = dart.clip_grad_norm(g, float("inf"), scale=0.5, out=out)
        assert float(n) == float("inf")
        for b, o in zip(before, g if out is None else out):
            assert np.array_equal(f64(o), 0.5 * b)   # (halves of small whole numbers: exact)
        g = [torch.ones(500, device="cuda"), torch.ones(10, device="cuda")]
        g[1][3] = float("nan")
        assert bool(torch.isnan(dart.clip_grad_norm(g, float("inf")))) and all(bool(torch.isnan(t).all()) for t in g)
