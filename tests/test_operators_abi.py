"""Refusals of the entry points around the blocks (norm, log probabilities,
gradient clipping): every check runs on the host before a launch, so these
need no GPU; the pointers are never used."""
import ctypes

import pytest

from paper_2608_02032_amd import dart

INVALID, UNSUPPORTED = 1, 2
F32, BF16 = 0, 1
P = 1 << 20  # a pointer of nothing; arguments a mebibyte apart do not meet


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(dart.LIB_PATH):
        pytest.skip("libdart.so not built")
    return dart.load_library()


def norm(lib, rows=4, dim=64, dtype=BF16, center=1, x=P, xs=64, res=2 * P, rs=64, w=3 * P, b=4 * P, eps=1e-6, out=5 * P,
         total=6 * P):
    return lib.dart_layernorm(rows, dim, dtype, center, x, xs, res, rs, w, b, eps, out, total, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), INVALID), (dict(dim=0), INVALID), (dict(dim=16385, xs=20000, rs=20000), UNSUPPORTED),
    (dict(center=2), INVALID), (dict(dtype=2), INVALID), (dict(xs=63), INVALID), (dict(rs=63), INVALID), (dict(rs=0), INVALID),
    (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(x=None), INVALID), (dict(out=None), INVALID),
    (dict(res=None), INVALID),                       # a sum without a residual
    (dict(rows=1 << 60), UNSUPPORTED), (dict(xs=1 << 60), UNSUPPORTED), (dict(rs=1 << 60), UNSUPPORTED),
    (dict(out=P + 2), INVALID), (dict(total=2 * P - 2), INVALID), (dict(out=6 * P), INVALID), (dict(out=6 * P + 16), INVALID),
    (dict(out=P, xs=72), INVALID),                   # in place needs dense rows
    (dict(total=2 * P, rs=72), INVALID), (dict(out=3 * P), INVALID), (dict(total=4 * P + 64), INVALID)])
def test_layernorm_refuses(lib, kw, status):
    assert norm(lib, **kw) == status
    assert lib.dart_last_error()


def norm_bwd(lib, rows=4, dim=64, dtype=BF16, gdtype=F32, center=1, x=P, xs=64, w=2 * P, eps=1e-6, dout=3 * P, dsum=4 * P,
             dx=5 * P, dw=6 * P, db=7 * P, ws=8 * P, nbytes=None):
    if nbytes is None:
        nbytes = max(256, lib.dart_layernorm_bwd_workspace_bytes(rows, dim))
    return lib.dart_layernorm_bwd(rows, dim, dtype, gdtype, center, x, xs, w, eps, dout, dsum, dx, dw, db, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), INVALID), (dict(dim=0), INVALID), (dict(dim=16385, xs=20000), UNSUPPORTED), (dict(center=-1), INVALID),
    (dict(dtype=3), INVALID), (dict(gdtype=2), INVALID), (dict(dtype=F32, gdtype=BF16), UNSUPPORTED), (dict(xs=10), INVALID),
    (dict(eps=-1.0), INVALID), (dict(x=None), INVALID), (dict(dout=None), INVALID), (dict(dx=None), INVALID),
    (dict(ws=None), INVALID), (dict(nbytes=0), INVALID), (dict(ws=8 * P + 4), INVALID), (dict(dx=P), INVALID),
    (dict(dx=3 * P + 16), INVALID), (dict(dw=2 * P), INVALID), (dict(dw=7 * P + 4), INVALID), (dict(db=5 * P), INVALID)])
def test_layernorm_bwd_refuses(lib, kw, status):
    assert norm_bwd(lib, **kw) == status
    assert lib.dart_last_error()


def lp(lib, rows=4, vocab=100, stride=104, dtype=BF16, logits=P, targets=2 * P, k=3, logprob=3 * P, ids=4 * P, tops=5 * P,
       ws=6 * P, nbytes=1 << 30):
    return lib.dart_token_logprobs(rows, vocab, stride, dtype, logits, targets, -100, k, logprob, 7 * P, 8 * P, 9 * P, ids, tops,
                                   ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), INVALID), (dict(vocab=0), INVALID), (dict(vocab=1 << 31, stride=1 << 31), UNSUPPORTED),
    (dict(vocab=(1 << 24) + 1, stride=1 << 25), UNSUPPORTED), (dict(stride=99), INVALID),
    (dict(dtype=-1), INVALID), (dict(k=-1), INVALID), (dict(k=101), INVALID), (dict(k=33), UNSUPPORTED), (dict(vocab=2, k=3), INVALID),
    (dict(logits=None), INVALID), (dict(targets=None), INVALID), (dict(ids=None), INVALID), (dict(tops=None), INVALID),
    (dict(rows=1 << 60), UNSUPPORTED)])
def test_token_logprobs_refuses(lib, kw, status):
    assert lp(lib, **kw) == status
    assert lib.dart_last_error()


def test_token_logprobs_refuses_a_small_workspace(lib):
    shape = dict(rows=1, vocab=200000, stride=200000, k=20)
    need = lib.dart_token_logprobs_workspace_bytes(1, 200000, BF16, 20)
    if need:
        assert lp(lib, nbytes=need - 1, **shape) == INVALID
        assert lp(lib, ws=None, nbytes=0, **shape) == INVALID
        assert lp(lib, ws=6 * P + 8, **shape) == INVALID
    assert lib.dart_token_logprobs_workspace_bytes(-1, 10, BF16, 0) == 0
    assert lib.dart_token_logprobs_workspace_bytes(1, 10, BF16, 11) == 0


def lp_bwd(lib, rows=4, vocab=100, stride=100, dtype=BF16, gdtype=BF16, logits=P, targets=2 * P, m=3 * P, ls=4 * P, ent=5 * P,
           dlp=6 * P, dent=7 * P, dl=8 * P, ds=100):
    return lib.dart_token_logprobs_bwd(rows, vocab, stride, dtype, gdtype, logits, targets, -100, m, ls, ent, dlp, dent, None, dl,
                                       ds, None)


def lp_grad(lib, rows=4, vocab=100, stride=100, dtype=BF16, gdtype=BF16, logits=P, targets=2 * P, m=3 * P, ls=4 * P, ent=5 * P,
            dlp=6 * P, dent=7 * P, dl=8 * P, ds=100, k=0):
    return lib.dart_token_logprobs_grad(rows, vocab, stride, dtype, gdtype, logits, targets, -100, k, dlp, dent, None, None, ent, m,
                                        ls, None, None, dl, ds, 9 * P, 1 << 30, None)


@pytest.mark.parametrize("fn", [lp_bwd, lp_grad])
@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), INVALID), (dict(vocab=0), INVALID), (dict(stride=99), INVALID), (dict(ds=99), INVALID),
    (dict(gdtype=4), INVALID), (dict(dtype=F32), UNSUPPORTED), (dict(logits=None), INVALID), (dict(targets=None), INVALID),
    (dict(m=None), INVALID), (dict(ls=None), INVALID), (dict(ent=None), INVALID), (dict(dl=None), INVALID),
    (dict(dl=P, gdtype=F32), INVALID), (dict(dl=P, stride=104), INVALID), (dict(dl=P + 2), INVALID)])
def test_token_logprobs_gradients_refuse(lib, fn, kw, status):
    assert fn(lib, **kw) == status
    assert lib.dart_last_error()


def clip(lib, grads=(P, 2 * P), outs=None, numels=(100, 50), dtypes=(F32, BF16), odtypes=None, max_norm=1.0, scale=1.0,
         norm=9 * P, ws=10 * P, nbytes=1 << 20, n=None, reads_only=False):
    n = len(grads) if n is None else n
    size = max(1, len(grads))
    g = (ctypes.c_void_p * size)(*grads)
    o = (ctypes.c_void_p * size)(*(grads if outs is None else outs))
    c = (ctypes.c_int64 * size)(*numels)
    d = (ctypes.c_int32 * size)(*dtypes)
    od = (ctypes.c_int32 * size)(*(dtypes if odtypes is None else odtypes))
    if reads_only:
        return lib.dart_grad_norm(n, g, c, d, scale, norm, ws, nbytes, None)
    return lib.dart_clip_grad_norm(n, g, o, c, d, od, max_norm, scale, norm, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(n=(1 << 24) + 1), UNSUPPORTED), (dict(numels=(100, -1)), INVALID),
    (dict(numels=(1 << 43, 1)), INVALID), (dict(numels=(1 << 42, 1 << 42)), INVALID),
    (dict(dtypes=(F32, 2)), INVALID), (dict(grads=(P, None)), INVALID),
    (dict(grads=(P, 2 * P + 1)), INVALID), (dict(grads=(P + 2, 2 * P)), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(norm=None), INVALID), (dict(ws=None), INVALID), (dict(nbytes=16), INVALID),
    (dict(ws=10 * P + 8), INVALID)])
def test_gradient_norm_and_clipping_refuse(lib, kw, status):
    assert clip(lib, **kw) == status
    assert lib.dart_last_error()
    assert clip(lib, reads_only=True, **kw) == status


@pytest.mark.parametrize("kw", [
    dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(outs=(P, None)), dict(odtypes=(F32, 5)), dict(outs=(P + 1, 2 * P)),
    dict(grads=(P, P), dtypes=(F32, F32)),                                    # the same tensor twice
    dict(grads=(P, P + 200), dtypes=(BF16, BF16), numels=(101, 50)),          # two that overlap
    dict(outs=(P + 4, 2 * P)), dict(outs=(P, 2 * P), odtypes=(BF16, BF16)),   # its own gradient, shifted or of another type
    dict(outs=(3 * P, 3 * P + 100)), dict(outs=(2 * P, 3 * P)),               # another output, another gradient
    dict(outs=(2 * P + 96, 3 * P))])
def test_clipping_refuses_outputs(lib, kw):
    assert clip(lib, **kw) == INVALID
    assert lib.dart_last_error()


def test_the_same_tensor_twice_may_be_read(lib):
    # past every other check only the workspace's size is left to refuse
    assert clip(lib, grads=(P, P), dtypes=(F32, F32), reads_only=True, nbytes=0) == INVALID
    assert b"workspace" in lib.dart_last_error()


def test_binding_refuses_what_is_not_on_the_gpu():
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="GPU"):
        dart.layernorm(x)
    with pytest.raises(ValueError, match="GPU"):
        dart.layernorm_bwd(x, x)
    with pytest.raises(ValueError, match="GPU"):
        dart.token_logprobs(x)
    with pytest.raises(ValueError, match="GPU"):
        dart.token_logprobs_grad(x, None, None)
    with pytest.raises(ValueError, match="GPU"):
        dart.clip_grad_norm([x], 1.0)
    with pytest.raises(TypeError):
        dart.layernorm(x.double())


def test_row_strides_and_dense_tensors():
    import torch
    a = torch.zeros(6, 5, 16)
    assert dart._row_stride(a[..., :12], "a") == 16
    assert dart._row_stride(a[:, :1, :12], "a") == 80       # one row in every five
    assert dart._row_stride(a[:1, :1, 3:9], "a") == 6       # one row: its own length
    assert dart._row_stride(torch.zeros(7), "a") == 7
    for bad in (a[:, :4, :12], a.transpose(1, 2), a[:, :, ::2]):
        with pytest.raises(ValueError):
            dart._row_stride(bad, "a")
    assert dart._row_stride(a[:, 0, :].expand(6, 16)[:1].expand(4, 16), "a") == 0   # refused by the library
    assert dart._dense(a.transpose(0, 2)) and dart._dense(a[2:4]) and dart._dense(torch.zeros(0, 3).t())
    assert not dart._dense(a[:, :4]) and not dart._dense(a[0, :1].expand(3, 16)) and not dart._dense(a[:, ::2].transpose(0, 1))


@pytest.mark.parametrize("vocab", [1, 2048, 2049, 50257, 131073, 1 << 24])
def test_no_rows_need_no_workspace(lib, vocab):
    for dtype in (F32, BF16):
        for k in (0, 1):
            assert lib.dart_token_logprobs_workspace_bytes(0, vocab, dtype, k) == 0
    # past every check there is nothing to launch
    assert lp(lib, rows=0, vocab=vocab, stride=vocab, k=0, logits=None, targets=None, logprob=None, ids=None, tops=None, ws=None,
              nbytes=0) == 0
    assert lp_bwd(lib, rows=0, vocab=vocab, stride=vocab, ds=vocab) == 0
    assert lp_grad(lib, rows=0, vocab=vocab, stride=vocab, ds=vocab) == 0


def test_norm_backward_refuses_a_workspace_in_its_arguments(lib):
    need = lib.dart_layernorm_bwd_workspace_bytes(4, 64)
    for k in range(1, 8):
        # it ends inside the argument at k P, or begins there
        assert norm_bwd(lib, ws=k * P) == INVALID and b"workspace overlaps" in lib.dart_last_error()
        assert norm_bwd(lib, ws=k * P - need + 16) == INVALID and b"workspace overlaps" in lib.dart_last_error()


LP = dict(logits=P, targets=2 * P, dlp=3 * P, dent=4 * P, dlse=5 * P, logprob=6 * P, ent=7 * P, m=8 * P, ls=9 * P, ids=10 * P,
          tops=11 * P, dl=12 * P, ws=14 * P)


def lp_apart(lib, one_call, rows=2, vocab=200000, k=3, **kw):
    a = dict(LP, **kw)
    need = lib.dart_token_logprobs_workspace_bytes(rows, vocab, BF16, k)
    assert need > 0
    if one_call:
        return lib.dart_token_logprobs_grad(rows, vocab, vocab, BF16, BF16, a["logits"], a["targets"], -100, k, a["dlp"], a["dent"],
                                            a["dlse"], a["logprob"], a["ent"], a["m"], a["ls"], a["ids"], a["tops"], a["dl"], vocab,
                                            a["ws"], need, None)
    return lib.dart_token_logprobs(rows, vocab, vocab, BF16, a["logits"], a["targets"], -100, k, a["logprob"], a["ent"], a["m"],
                                   a["ls"], a["ids"], a["tops"], a["ws"], need, None)


@pytest.mark.parametrize("one_call", [False, True])
@pytest.mark.parametrize("name", ["logprob", "ent", "m", "ls", "ids", "tops", "ws"])
def test_token_logprobs_results_meet_nothing_else(lib, one_call, name):
    others = [n for n in LP if n != name and (one_call or n not in ("dlp", "dent", "dlse", "dl"))]
    for other in others:
        assert lp_apart(lib, one_call, **{name: LP[other]}) == INVALID and b"overlaps" in lib.dart_last_error(), other
    # the last byte of the logits and, in the one call, of their gradient
    end = 2 * 200000 * 2
    assert lp_apart(lib, one_call, **{name: P + end - 16}) == INVALID and b"overlaps" in lib.dart_last_error()
    if one_call:
        assert lp_apart(lib, True, **{name: 12 * P + end - 16}) == INVALID and b"overlaps" in lib.dart_last_error()


def test_gradient_of_the_logits_meets_no_input(lib):
    for other in ("targets", "dlp", "dent", "dlse"):
        assert lp_apart(lib, True, dl=LP[other]) == INVALID and b"dlogits" in lib.dart_last_error()
    for k in range(2, 8):
        assert lp_bwd(lib, dl=k * P) == INVALID and b"dlogits" in lib.dart_last_error()
        assert lp_bwd(lib, dl=k * P - 2 * 400 + 2) == INVALID and b"dlogits" in lib.dart_last_error()


@pytest.mark.parametrize("reads_only", [False, True])
def test_norm_and_workspace_lie_in_no_tensor(lib, reads_only):
    need = lib.dart_grad_norm_workspace_bytes(2)
    for kw in (dict(norm=P), dict(norm=P + 396), dict(norm=2 * P + 96), dict(ws=P), dict(ws=2 * P + 96), dict(ws=P - need + 16),
               dict(norm=10 * P), dict(norm=10 * P + need - 4)):
        assert clip(lib, reads_only=reads_only, **kw) == INVALID and b"overlaps" in lib.dart_last_error(), kw
    if not reads_only:
        for kw in (dict(norm=3 * P + 8), dict(ws=4 * P)):
            assert clip(lib, outs=(3 * P, 4 * P), **kw) == INVALID and b"overlaps" in lib.dart_last_error(), kw
