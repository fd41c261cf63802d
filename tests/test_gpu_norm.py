"""Layer norm and RMS norm of the residual stream, forward and backward,
against the definition in 64 bits.

Bounds.  u = 2^-24 is half a step of float.  A sum of D products in any order
of partial sums here rounds fewer than 64 times along any path beside the
partial sums it meets (at most 64 elements in one lane, then trees), so the
mean is off by at most 64 u max|s| and everything of the deviations by that
over the row's deviation: relative to the row's largest output
64 u (1 + max|s| inv), taken four times (mean, mean square, product sums, the
formula's own few roundings).  A bf16 result adds half a step of its own, 2^-8 of it."""
import numpy as np
import pytest

from paper_2608_02032_amd import dart

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}
EPS = 1e-6


def tensor(a, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()


def f64(t):
    return t.detach().double().cpu().numpy()


def reference(x, res, w, b, center, dtype, eps=EPS):
    """(sum as stored, deviations, inv, out) in 64 bits."""
    s = f64(x) if res is None else f64((x.float() + res.float()).to(x.dtype))
    dev = s - s.mean(-1, keepdims=True) if center else s
    inv = 1 / np.sqrt((dev ** 2).mean(-1, keepdims=True) + eps)
    return s, dev, inv, dev * inv * (1 if w is None else f64(w)) + (0 if b is None else f64(b))


def condition(s, inv):
    return 4 * 64 * U * (1 + np.abs(s).max(-1, keepdims=True) * inv)


def within(got, ref, bound, what):
    got = f64(got)
    assert got.shape == ref.shape, what
    bad = ~(np.abs(got - ref) <= bound)
    print("  %-8s worst |d|/bound %.3f" % (what, float((np.abs(got - ref) / np.maximum(bound, 1e-300)).max()) if ref.size else 0), flush=True)
    assert not bad.any(), "%s: %d of %d outside, first at %s" % (what, bad.sum(), bad.size, np.argwhere(bad)[0])


def check_forward(x, res, w, b, center, dtype, out, total):
    s, dev, inv, ref = reference(x, res, w, b, center, dtype)
    if res is not None:
        assert np.array_equal(f64(total), s), "sum"
    scale = np.abs(dev * inv * (1 if w is None else f64(w))).max(-1, keepdims=True) + (0 if b is None else np.abs(f64(b)).max())
    within(out, ref, STEP[dtype] * np.abs(ref) + condition(s, inv) * scale, "out")
    return s, dev, inv


def check_backward(s, dev, inv, w, center, dout, dsum, g, gdtype):
    n = s.shape[-1]
    xh, do = dev * inv, f64(dout)
    gw = do * (1 if w is None else f64(w))
    m1 = gw.mean(-1, keepdims=True) if center else 0.0
    m2 = (gw * xh).mean(-1, keepdims=True)
    dx = inv * (gw - m1 - xh * m2) + (0 if dsum is None else f64(dsum))
    c = condition(s, inv)
    scale = inv * (np.abs(gw).max(-1, keepdims=True) + np.abs(gw).mean(-1, keepdims=True)
                   + np.abs(xh).max(-1, keepdims=True) * np.abs(gw * xh).mean(-1, keepdims=True))
    scale = scale + (0 if dsum is None else np.abs(f64(dsum)))
    within(g["dx"], dx, STEP[gdtype] * np.abs(dx) + c * scale, "dx")
    # sums over the rows: at most 64 rows and 64 partial sums in one thread, then trees
    rows = (-1, n)
    if g["dweight"] is not None:
        t = (do * xh).reshape(rows)
        e = (np.abs(do) * (np.abs(xh) + np.abs(xh).max(-1, keepdims=True)) * c).reshape(rows)
        within(g["dweight"], t.sum(0), 256 * U * np.abs(t).sum(0) + e.sum(0) + 1e-30, "dweight")
    if g["dbias"] is not None:
        t = do.reshape(rows)
        within(g["dbias"], t.sum(0), 256 * U * np.abs(t).sum(0) + 1e-30, "dbias")


def rand(rng, *shape, shift=0.0):
    return rng.standard_normal(shape) + shift


# widths: one, odd, each side of the vectors, of a wave's and a workgroup's pieces, the widest
DIMS = [1, 2, 7, 64, 65, 127, 256, 512, 513, 768, 1000, 1001, 1024, 1025, 2048, 2056, 4096, 5000, 8192, 8200, 12289, 16384]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", DIMS)
def test_widths(dtype, D):
    rng = np.random.default_rng(D)
    rows = 5 if D > 2048 else 37
    for center, use_res, use_w, use_b in [(True, True, True, True), (False, False, True, False), (True, False, False, True)]:
        print("\n[gpu-case] norm %s rows=%d D=%d center=%d res=%d w=%d b=%d" % (dtype, rows, D, center, use_res, use_w, use_b), flush=True)
        x = tensor(rand(rng, rows, D, shift=0.5), dtype)
        res = tensor(rand(rng, rows, D), dtype) if use_res else None
        w = tensor(1 + 0.2 * rand(rng, D), "fp32") if use_w else None
        b = tensor(rand(rng, D), "fp32") if use_b else None
        r = dart.layernorm(x, w, b, residual=res, eps=EPS, center=center)
        out, total = r if use_res else (r, x)
        s, dev, inv = check_forward(x, res, w, b, center, dtype, out, total)
        for gdtype in {"fp32", dtype}:
            dout = tensor(rand(rng, rows, D, shift=0.1), gdtype)
            dsum = tensor(rand(rng, rows, D), gdtype) if use_res else None
            g = dart.layernorm_bwd(total, dout, w, dsum=dsum, eps=EPS, center=center, want_bias=use_b)
            assert (g["dweight"] is None) == (w is None) and (g["dbias"] is None) == (b is None)
            check_backward(s, dev, inv, w, center, dout, dsum, g, gdtype)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 31, 33, 64, 255, 257, 1023, 2049, 4099, 20000])
@pytest.mark.parametrize("D", [24, 768, 2304])
def test_rows(rows, D):
    rng = np.random.default_rng(rows * 7 + D)
    print("\n[gpu-case] norm rows=%d D=%d" % (rows, D), flush=True)
    x, res, dout, dsum = (tensor(rand(rng, rows, D), "bf16") for _ in range(4))
    w, b = tensor(rand(rng, D), "fp32"), tensor(rand(rng, D), "fp32")
    out, total = dart.layernorm(x, w, b, residual=res, eps=EPS)
    s, dev, inv = check_forward(x, res, w, b, True, "bf16", out, total)
    check_backward(s, dev, inv, w, True, dout, dsum, dart.layernorm_bwd(total, dout, w, dsum=dsum, eps=EPS, want_bias=True), "bf16")


def test_no_rows():
    import torch
    x = torch.empty(0, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    out, s = dart.layernorm(x, w, residual=x)
    assert out.shape == (0, 64) and s.shape == (0, 64)
    g = dart.layernorm_bwd(x, x, w, want_bias=True)
    torch.cuda.synchronize()
    assert g["dx"].shape == (0, 64) and not g["dweight"].any() and not g["dbias"].any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D,pad,first", [(64, 64, 0), (768, 8, 8), (768, 5, 0), (768, 5, 3), (100, 4, 2), (1001, 7, 1), (8191, 1, 1)])
def test_strides_and_alignment(dtype, D, pad, first):
    """Rows out of a wider tensor, and buffers that begin anywhere; what lies between is left as it was."""
    import torch
    print("\n[gpu-case] norm stride %s D=%d pad=%d first=%d" % (dtype, D, pad, first), flush=True)
    rng = np.random.default_rng(D + pad)
    rows = 13
    wide = tensor(rand(rng, rows, D + pad + first), dtype)
    x = wide[:, first:first + D]
    res = tensor(rand(rng, rows * D + 3), dtype)[3:].view(rows, D)
    w = tensor(rand(rng, D + 1), "fp32")[1:]
    b = tensor(rand(rng, D + 2), "fp32")[2:]
    obuf = torch.full((rows * D + 16,), 7.0, dtype=x.dtype, device="cuda")
    sbuf = torch.full((rows * D + 16,), 7.0, dtype=x.dtype, device="cuda")
    out, total = obuf[first:first + rows * D].view(rows, D), sbuf[1:1 + rows * D].view(rows, D)
    dart.layernorm(x, w, b, residual=res, eps=EPS, out=out, sum_out=total)
    s, dev, inv = check_forward(x, res, w, b, True, dtype, out, total)
    for buf, at in ((obuf, first), (sbuf, 1)):
        edge = torch.cat([buf[:at], buf[at + rows * D:]])
        assert bool((edge == 7.0).all())
    dout = tensor(rand(rng, rows * D + 1), dtype)[1:].view(rows, D)
    dbuf = torch.full((rows * D + 16,), 7.0, dtype=x.dtype, device="cuda")
    g = dart.layernorm_bwd(total, dout, w, eps=EPS, want_bias=True, dx=dbuf[5:5 + rows * D].view(rows, D))
    check_backward(s, dev, inv, w, True, dout, None, g, dtype)
    assert bool((torch.cat([dbuf[:5], dbuf[5 + rows * D:]]) == 7.0).all())
    # the backward at a slice of a wider tensor
    s2, dev2, inv2, _ = reference(x, None, w, None, False, dtype)
    check_backward(s2, dev2, inv2, w, False, dout, None, dart.layernorm_bwd(x, dout, w, eps=EPS, center=False), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 1001, 4096])
def test_in_place(dtype, D):
    rng = np.random.default_rng(D)
    print("\n[gpu-case] norm in place %s D=%d" % (dtype, D), flush=True)
    x0, r0 = tensor(rand(rng, 19, D), dtype), tensor(rand(rng, 19, D), dtype)
    w = tensor(rand(rng, D), "fp32")
    ref, sref = dart.layernorm(x0, w, residual=r0, eps=EPS)
    for into in ("residual", "x", "both"):
        x, r = x0.clone(), r0.clone()
        out, total = dart.layernorm(x, w, residual=r, eps=EPS, sum_out=x if into == "x" else r, out=x if into == "both" else None)
        assert out.equal(ref) and total.equal(sref)
    x = x0.clone()
    assert dart.layernorm(x, w, eps=EPS, out=x).equal(dart.layernorm(x0, w, eps=EPS))
    dout, dsum = tensor(rand(rng, 19, D), dtype), tensor(rand(rng, 19, D), dtype)
    g = dart.layernorm_bwd(sref, dout, w, dsum=dsum, eps=EPS)
    for into in (0, 1):
        a, b = dout.clone(), dsum.clone()
        h = dart.layernorm_bwd(sref, a, w, dsum=b, eps=EPS, dx=(a, b)[into])
        assert h["dx"].equal(g["dx"]) and h["dweight"].equal(g["dweight"])


def test_large_mean_and_constant_rows():
    """The deviations are small against the mean; a row without any has out = bias and a finite gradient."""
    rng = np.random.default_rng(5)
    D = 1024
    a = rand(rng, 8, D, shift=300.0)
    a[3] = 2.5
    a[4] = 0.0
    x, w, b = tensor(a, "fp32"), tensor(rand(rng, D), "fp32"), tensor(rand(rng, D), "fp32")
    out = dart.layernorm(x, w, b, eps=EPS)
    s, dev, inv = check_forward(x, None, w, b, True, "fp32", out, x)
    assert np.array_equal(f64(out)[3], f64(b)) and np.array_equal(f64(out)[4], f64(b))
    dout = tensor(rand(rng, 8, D), "fp32")
    g = dart.layernorm_bwd(x, dout, w, eps=EPS, want_bias=True)
    check_backward(s, dev, inv, w, True, dout, None, g, "fp32")


@pytest.mark.parametrize("D", [64, 1000, 8192])
def test_nonfinite_rows_stay_alone(D):
    import torch
    rng = np.random.default_rng(D)
    a = rand(rng, 9, D)
    x = tensor(a, "bf16")
    bad = x.clone()
    bad[2, D // 2], bad[5, 0], bad[7, D - 1] = float("nan"), float("inf"), float("-inf")
    w = tensor(rand(rng, D), "fp32")
    dout = tensor(rand(rng, 9, D), "bf16")
    ok = [0, 1, 3, 4, 6, 8]
    for center in (True, False):
        y, z = dart.layernorm(x, w, center=center), dart.layernorm(bad, w, center=center)
        assert y[ok].equal(z[ok]) and bool(torch.isnan(z[2]).all())
        assert bool(torch.isnan(z[[5, 7]]).any(1).all())
        g, h = dart.layernorm_bwd(x, dout, w, center=center)["dx"], dart.layernorm_bwd(bad, dout, w, center=center)["dx"]
        assert g[ok].equal(h[ok]) and bool(torch.isnan(h[2]).all())


def test_gradient_against_differences():
    """d loss / d x, d weight, d bias by central differences of the 64-bit forward, loss = sum(dout out) + sum(dsum s)."""
    rng = np.random.default_rng(11)
    R, D = 3, 20
    x, w, b, dout, dsum = rand(rng, R, D), rand(rng, D), rand(rng, D), rand(rng, R, D), rand(rng, R, D)
    x, w, b, dout, dsum = (a.astype(np.float32).astype(np.float64) for a in (x, w, b, dout, dsum))

    def loss(x, w, b, center):
        dev = x - x.mean(-1, keepdims=True) if center else x
        return (dout * (dev / np.sqrt((dev ** 2).mean(-1, keepdims=True) + EPS) * w + b)).sum() + (dsum * x).sum()

    h = 1e-5   # central differences: h^2 of third derivatives (of order 10 here), 1e-16 / h of rounding
    for center in (True, False):
        g = dart.layernorm_bwd(tensor(x, "fp32"), tensor(dout, "fp32"), tensor(w, "fp32"), dsum=tensor(dsum, "fp32"), eps=EPS,
                               center=center, want_bias=True)
        for k, got in ((0, g["dx"]), (1, g["dweight"]), (2, g["dbias"])):
            args = [x, w, b]
            num = np.zeros_like(args[k])
            for i in np.ndindex(num.shape):
                p, q = [a.copy() for a in args], [a.copy() for a in args]
                p[k][i] += h
                q[k][i] -= h
                num[i] = (loss(*p, center) - loss(*q, center)) / (2 * h)
            assert np.abs(f64(got) - num).max() <= 2e-5 * max(1.0, np.abs(num).max())


def test_other_stream_and_device_checks():
    import torch
    rng = np.random.default_rng(3)
    x, w = tensor(rand(rng, 500, 768), "bf16"), tensor(rand(rng, 768), "fp32")
    dout = tensor(rand(rng, 500, 768), "bf16")
    ref, gref = dart.layernorm(x, w), dart.layernorm_bwd(x, dout, w)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):
        out, g = dart.layernorm(x, w, stream=side), dart.layernorm_bwd(x, dout, w, stream=side)
        junk = [torch.full((1 << 20,), 3.0, device="cuda") for _ in range(8)]   # what the calls' workspaces must not be
    side.synchronize()
    assert out.equal(ref) and g["dx"].equal(gref["dx"]) and g["dweight"].equal(gref["dweight"]) and junk
    with pytest.raises(ValueError):
        dart.layernorm(x, w.cpu())
    with pytest.raises(ValueError):
        dart.layernorm(x, w[:5])
    with pytest.raises(ValueError):
        dart.layernorm(x, w, residual=x.float())
    with pytest.raises(ValueError):
        dart.layernorm(x[:1].expand(500, 768), w, out=x.view(-1)[:5])
    with pytest.raises(dart.DartError):
        dart.layernorm(x[:1].expand(500, 768), w)
    with pytest.raises(dart.DartError):
        dart.layernorm_bwd(x.float(), dout, w)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [1000, 1030, 1500, 1536, 1700, 2047, 2048])
def test_many_rows_of_a_wave(dtype, D):
    """Enough rows for a wave each, and for workgroups of several rounds."""
    rng = np.random.default_rng(D)
    for rows in (1024, 4100):
        print("\n[gpu-case] norm %s rows=%d D=%d" % (dtype, rows, D), flush=True)
        x, res = tensor(rand(rng, rows, D, shift=0.5), dtype), tensor(rand(rng, rows, D), dtype)
        w, b = tensor(1 + 0.2 * rand(rng, D), "fp32"), tensor(rand(rng, D), "fp32")
        out, total = dart.layernorm(x, w, b, residual=res, eps=EPS)
        s, dev, inv = check_forward(x, res, w, b, True, dtype, out, total)
        for gdtype in {"fp32", dtype}:
            dout, dsum = tensor(rand(rng, rows, D), gdtype), tensor(rand(rng, rows, D), gdtype)
            g = dart.layernorm_bwd(total, dout, w, dsum=dsum, eps=EPS, want_bias=True)
            check_backward(s, dev, inv, w, True, dout, dsum, g, gdtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [3, 100, 1000, 1001, 1500, 2047, 4095, 5000, 8191, 12289, 16384])
def test_constant_rows_of_any_width(dtype, D):
    """A row of one value has no deviation: out = bias to the last bit, xh = 0 and inv = eps^-1/2.  Of values of eight
    bits every partial sum of up to 2^14 has 22 and is exact in float, so that only the division could round."""
    rng = np.random.default_rng(D)
    print("\n[gpu-case] norm constant rows %s D=%d" % (dtype, D), flush=True)
    c = np.array([300.0, 2.5, 3.0, 0.1, -1234.5, 1.0 / 3.0, 0.0, 77.7])
    x = tensor(f64(tensor(np.repeat(c[:, None], D, 1), "bf16")), dtype)
    w, b = tensor(rand(rng, D), "fp32"), tensor(rand(rng, D), "fp32")
    out = dart.layernorm(x, w, b, eps=EPS)
    want = b.to(x.dtype).double().cpu().numpy()
    assert np.array_equal(f64(out), np.broadcast_to(want, out.shape))
    zero = x.new_zeros(x.shape)
    assert np.array_equal(f64(dart.layernorm(x, w, b, residual=zero, eps=EPS)[0]), np.broadcast_to(want, out.shape))
    for gdtype in {"fp32", dtype}:
        dout = tensor(rand(rng, len(c), D), gdtype)
        g = dart.layernorm_bwd(x, dout, w, eps=EPS, want_bias=True)
        inv = 1 / np.sqrt(EPS)
        gw = f64(dout) * f64(w)
        dx = inv * (gw - gw.mean(-1, keepdims=True))
        # the sum of the gradients (fewer than 64 roundings along a path) and the formula's few
        bound = 2 * 64 * U * inv * np.abs(gw).max(-1, keepdims=True)
        within(g["dx"], dx, STEP[gdtype] * np.abs(dx) + bound, "dx")
        assert not bool(g["dweight"].any())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [1000, 4095, 16384])
def test_small_deviations_from_a_large_mean(dtype, D):
    """Rows that leave one value by a step of bfloat16 in places (sums exact, as above): out is off by the mean's one
    rounding, u |c| inv, and by the mean square's (fewer than 64 along a path): 128 u of the row's largest."""
    rng = np.random.default_rng(D + 1)
    print("\n[gpu-case] norm small deviations %s D=%d" % (dtype, D), flush=True)
    c = np.array([300.0, 3.0, -40.0, 1000.0])[:, None]
    a = np.broadcast_to(c, (4, D)) * (1 + (rng.random((4, D)) < 0.2) * 2.0 ** -7)
    x = tensor(f64(tensor(a, "bf16")), dtype)
    w = tensor(1 + 0.1 * rand(rng, D), "fp32")
    for center in (True, False):
        s, dev, inv, ref = reference(x, None, w, None, center, dtype)
        bound = 2 * U * np.abs(s).max(-1, keepdims=True) * inv + 128 * U * np.abs(dev * inv).max(-1, keepdims=True)
        bound = STEP[dtype] * np.abs(ref) + bound * float(w.max())
        within(dart.layernorm(x, w, eps=EPS, center=center), ref, bound, "out")
