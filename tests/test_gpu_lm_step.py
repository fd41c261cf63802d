"""The steps around the blocks as a training step and a scoring pass run them
together: residual addition and norm, log probabilities with their gradient,
clipping; through layer.py, in one captured graph, and against 64 bits.

Bounds: each operator's own tests hold it to its rounding; a chain of them,
each step's rounding at most 2^-24 of values that sums and norms keep at their
size, stays within a few hundred of that relative to the largest (products of
K terms add sqrt(K))."""
import numpy as np
import pytest

from paper_2608_02032_amd import dart

pytestmark = pytest.mark.gpu

REL = 2e-5   # 300 half steps of float, relative to the largest


def near(got, ref, rel=REL, what=""):
    got, ref = got.detach().double().cpu(), ref.detach().double().cpu()
    d, m = float((got - ref).abs().max()), float(ref.abs().max())
    print("  %-12s %.2e of the largest" % (what, d / m if m else d), flush=True)
    assert d <= rel * m + 1e-30, what


def test_residual_stream_head_and_loss_against_64_bits():
    """Two additions with their norms, a head, log probabilities and entropies: outputs and every gradient."""
    import torch
    from paper_2608_02032_amd import layer
    torch.manual_seed(0)
    B, L, D, V = 3, 17, 96, 130
    base = {"u": torch.randn(B, L, D), "d1": torch.randn(B, L, D), "d2": torch.randn(B, L, D),
            "w1": 1 + 0.1 * torch.randn(D), "w2": 1 + 0.1 * torch.randn(D), "head": torch.randn(V, D) * D ** -0.5}
    t = torch.randint(0, V, (B, L))
    t[:, ::4] = -100
    wt = torch.rand(B, L)

    def run(p, ops):
        s, n1 = ops["add_norm"](p["u"], p["d1"], p["w1"])
        s, n2 = ops["add_norm"](s, p["d2"] * n1, p["w2"])
        logits = n2 @ p["head"].t() + 0.1 * (s @ p["head"].t())
        lp, ent = ops["logprobs"](logits)
        return -(wt.to(lp) * lp).sum() - 0.05 * ent.sum(), lp, ent

    def add_norm64(u, d, w):
        s = u + d
        return s, s * torch.rsqrt((s * s).mean(-1, keepdim=True) + 1e-6) * w

    def logprobs64(l):
        q = torch.log_softmax(l, -1)
        has = t != -100
        return torch.where(has, q.gather(-1, t.clamp(min=0)[..., None])[..., 0], torch.zeros((), dtype=l.dtype)), -(q.exp() * q).sum(-1)

    p64 = {k: v.double().requires_grad_() for k, v in base.items()}
    ref = run(p64, {"add_norm": add_norm64, "logprobs": logprobs64})
    ref[0].backward()
    p = {k: v.clone().cuda().requires_grad_() for k, v in base.items()}
    got = run(p, {"add_norm": layer.add_norm, "logprobs": lambda l: layer.token_logprobs(l, t.cuda())})
    got[0].backward()
    for k, a, b in zip(("loss", "logprob", "entropy"), got, ref):
        near(a, b, what=k)
    for k in base:
        near(p[k].grad, p64[k].grad, what="d" + k)


def test_unused_outputs_have_no_gradient():
    import torch
    from paper_2608_02032_amd import layer
    u, d = (torch.randn(5, 64, device="cuda").requires_grad_() for _ in range(2))
    w = torch.ones(64, device="cuda").requires_grad_()
    s, n = layer.add_norm(u, d, w)
    s.sum().backward(retain_graph=True)
    assert bool((u.grad == 1).all()) and bool((d.grad == 1).all()) and w.grad is None
    u.grad = d.grad = None
    n.sum().backward()
    assert u.grad.equal(d.grad) and u.grad is not d.grad and u.grad.data_ptr() != d.grad.data_ptr() and w.grad is not None
    l = torch.randn(4, 9, device="cuda").requires_grad_()
    lp, ent = layer.token_logprobs(l, torch.arange(4, device="cuda"))
    ent.sum().backward()
    q = torch.log_softmax(l.detach().double(), -1)
    near(l.grad, -(q.exp() * (q - (q.exp() * q).sum(-1, keepdim=True))), what="entropy")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_captured_step_replays_as_the_eager_one(dtype):
    """Norm with addition, loss with gradient, norm backward and clipping in one graph, replayed with new inputs
    between eager work: every replay gives what eager calls on the same inputs give."""
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    print("\n[gpu-case] captured step %s" % dtype, flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    R, D, V = 70, 320, 5003

    def fresh():
        return {"x": torch.randn(R, D, generator=g, device="cuda").to(t), "res": torch.randn(R, D, generator=g, device="cuda").to(t),
                "dout": torch.randn(R, D, generator=g, device="cuda").to(t), "logits": (3 * torch.randn(R, V, generator=g, device="cuda")).to(t),
                "t": torch.randint(0, V, (R,), generator=g, device="cuda"), "dlp": torch.randn(R, generator=g, device="cuda"),
                "one": (3 * torch.randn(2, 90001, generator=g, device="cuda")).to(t)}

    w = 1 + 0.1 * torch.randn(D, generator=g, device="cuda")

    def step(s):
        out, total = dart.layernorm(s["x"], w, residual=s["res"], center=False)
        r = dart.token_logprobs_grad(s["logits"], s["t"], s["dlp"], dentropy=s["dlp"], top_k=3)
        few = dart.token_logprobs(s["one"], top_k=20)          # segments and their joining
        two = dart.token_logprobs_bwd(s["logits"], r["row_max"], r["log_sum"], targets=s["t"], dlogprob=s["dlp"])
        n = dart.layernorm_bwd(total, s["dout"], w, dsum=s["dout"], center=False, want_bias=True)
        grads = [n["dweight"], n["dbias"], n["dx"], r["dlogits"]]
        clipped = [torch.empty_like(v) for v in grads]
        norm = dart.clip_grad_norm(grads, 0.5, out=clipped)
        return [out, total, r["logprob"], r["entropy"], r["top_ids"], r["top_logprobs"], r["dlogits"], few["top_ids"], few["log_sum"],
                two, n["dx"], n["dweight"], n["dbias"], norm] + clipped

    static = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(static)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(static)
    for k in range(4):
        new = fresh()
        for name, v in new.items():
            static[name].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        ref = step(new)
        junk = torch.randn(1 << 20, device="cuda").sum()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(outs, ref)):
            assert a.equal(b), "replay %d output %d" % (k, i)
        assert bool(torch.isfinite(junk))


def test_many_tensors_in_a_captured_clip():
    """More tensors than travel in a launch's arguments: the table is written by the graph too."""
    import torch
    grads = [torch.randn(50 + k, device="cuda") for k in range(300)]
    out = [torch.empty_like(v) for v in grads]
    dart.clip_grad_norm(grads, 1.0, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = dart.clip_grad_norm(grads, 1.0, out=out)
    for k in range(3):
        for v in grads:
            v.normal_()
        graph.replay()
        torch.cuda.synchronize()
        want = dart.clip_grad_norm(grads, 1.0, out=[torch.empty_like(v) for v in grads])
        assert norm.equal(want)
        total = float(torch.cat(grads).double().norm())
        near(torch.cat(out), torch.cat(grads).double() / total, what="clipped")


def test_a_training_step_against_torch():
    """DartLM's loss, accuracy, gradients and clipping, against torch's own loss and clipping on the same logits."""
    import torch
    import torch.nn.functional as F
    from paper_2608_02032_amd import layer, mqar
    torch.manual_seed(3)
    vocab = mqar.MqarVocab(32, 32)
    model = layer.DartLM(vocab.size, 64, 2, 16, 16).cuda()
    tok, lab = mqar.mqar_batch(np.random.default_rng(0), 8, 128, 8, vocab)
    tok, lab = torch.from_numpy(tok).cuda(), torch.from_numpy(lab).cuda()
    params = [p for p in model.parameters()]
    logits = model(tok)
    ref_loss = F.cross_entropy(logits.view(-1, vocab.size), lab.view(-1), ignore_index=mqar.IGNORE)
    ref = torch.autograd.grad(ref_loss, params, retain_graph=True)
    m = lab != mqar.IGNORE
    r = dart.token_logprobs_grad(logits.detach(), lab, -m.float() / m.sum(), top_k=1, ignore_index=mqar.IGNORE)
    near(-r["logprob"].sum() / m.sum(), ref_loss, what="loss")
    assert r["top_ids"][..., 0][m].equal(logits.argmax(-1)[m])
    got = torch.autograd.grad(logits, params, r["dlogits"], retain_graph=True)
    lp, _ = layer.token_logprobs(logits, lab, ignore_index=mqar.IGNORE)
    two = torch.autograd.grad(-lp.sum() / m.sum(), params)
    for a, b, c in zip(got, two, ref):
        near(a, c, rel=1e-4, what="one call")   # the chain through two blocks' backward adds its own roundings
        near(b, c, rel=1e-4, what="two calls")
    for p, v in zip(params, ref):
        p.grad = v.clone()
    want = torch.nn.utils.clip_grad_norm_(params, 0.1)
    mine = [v.clone() for v in ref]
    norm = dart.clip_grad_norm(mine, 0.1)
    near(norm, want, what="norm")
    for a, p in zip(mine, params):
        near(a, p.grad, what="clipped")


def test_train_mqar_steps():
    """A few steps run and return finite losses and accuracies, the first one the untrained model's."""
    from paper_2608_02032_amd import layer, mqar
    losses, accs = layer.train_mqar(3, L=64, R=4, batch=4, vocab=mqar.MqarVocab(16, 16))
    assert len(losses) == len(accs) == 3 and np.all(np.isfinite(losses)) and all(0 <= a <= 1 for a in accs)


def test_a_second_derivative_is_refused():
    import torch
    from paper_2608_02032_amd import layer
    u = torch.randn(4, 32, device="cuda", requires_grad=True)
    w = torch.ones(32, device="cuda", requires_grad=True)
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    for f in (lambda: layer._Norm.apply(u, w), lambda: layer.add_norm(u, u, w)[1], lambda: layer.token_logprobs(u, t)[0]):
        g, = torch.autograd.grad(f().square().sum(), u, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            g.sum().backward()


def test_results_can_be_changed_in_place():
    """A loss masked in place, as training loops do: each result is a tensor of its own for autograd."""
    import torch
    from paper_2608_02032_amd import layer
    torch.manual_seed(4)
    l = torch.randn(6, 300, device="cuda", requires_grad=True)
    t = torch.arange(6, device="cuda") * 40
    wt = torch.rand(6, device="cuda")
    lp, ent = layer.token_logprobs(l, t)
    want, = torch.autograd.grad((lp * wt).sum() - 0.1 * ent.sum(), l)
    lp, ent = layer.token_logprobs(l, t)
    lp *= wt
    (lp.sum() - 0.1 * ent.sum()).backward()
    assert l.grad.equal(want)
    # what the backward needs of a result is still guarded
    lp, ent = layer.token_logprobs(l, t)
    ent *= 2
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        ent.sum().backward()
    # whatever the leading axes, none of them too
    for shape in ((300,), (2, 3, 300), (0, 300), (4, 0, 300)):
        l = torch.randn(shape, device="cuda", requires_grad=True)
        lp, ent = layer.token_logprobs(l, torch.zeros(shape[:-1], dtype=torch.int64, device="cuda"))
        lp *= 0.5
        (lp.sum() + ent.sum()).backward()
        assert lp.shape == ent.shape == shape[:-1] and l.grad.shape == shape


def test_residual_streams_that_the_norm_kernel_does_not_take():
    """A bfloat16 residual stream under float32 weights (promoted by the norm) and rows of more than 16384 channels."""
    import torch
    from paper_2608_02032_amd import layer
    torch.manual_seed(7)
    blk = layer.DartBlock(64, 16, 64, 2, 16).cuda()
    u = torch.randn(2, 48, 64, device="cuda").to(torch.bfloat16).requires_grad_()
    y = blk(u)
    assert y.dtype == torch.float32
    y.square().mean().backward()
    # the same stream in float32: the norm's bfloat16 roundings (the square, its mean, the reciprocal root, the product,
    # half a step 2^-8 each), times a block's gain, at most eight: every branch ends in a norm
    v = u.detach().float().requires_grad_()
    z = blk(v)
    z.square().mean().backward()
    near(y, z, rel=8 * 4 * 2.0 ** -8, what="bf16 stream")
    assert u.grad.dtype == torch.bfloat16 and bool(torch.isfinite(u.grad).all())
    D = 16384 + 64
    lm = layer.DartLM(24, D, n_layers=0).cuda()
    tok = torch.randint(0, 24, (2, 5), device="cuda")
    logits = lm(tok)
    logits.square().sum().backward()
    e = lm.emb.weight.detach().double()[tok]
    want = (e * torch.rsqrt(e.square().mean(-1, keepdim=True) + 1e-6)) @ lm.head.weight.detach().double().t()
    near(logits, want, rel=1e-4, what="wide")   # products of 16448 terms: sqrt of it, 128, half steps
    assert bool(lm.norm_w.grad.any())
