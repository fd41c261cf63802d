"""The residual stream's norm of the layer where the library's kernel does not
serve: rows of any width and type, on the host too, in torch."""
import pytest


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float64"])
@pytest.mark.parametrize("d", [1, 64, 16384 + 64])
def test_norm_of_the_residual_stream_on_the_host(dtype, d):
    import torch
    from paper_2608_02032_amd import layer
    t = getattr(torch, dtype)
    torch.manual_seed(d)
    lm = layer.DartLM(7, d, n_layers=0, headdim=2).to(t)
    tok = torch.randint(0, 7, (3, 4))
    out = lm(tok)
    out.float().sum().backward()
    e = lm.emb.weight.detach().double()[tok]
    want = (e * torch.rsqrt(e.square().mean(-1, keepdim=True) + 1e-6)) @ lm.head.weight.detach().double().t()
    # four roundings of the norm at half a step each, and sqrt(d) <= 129 of them in the head's sums
    assert out.shape == (3, 4, 7) and float((out.detach().double() - want).abs().max()) <= 64 * torch.finfo(t).eps * float(want.abs().max() + 1)
    assert lm.norm_w.grad.dtype == t
