"""Norm, recurrence, token loss and optimizer in a row, as a learner runs them (GPU)."""
import math

import pytest
import torch

from paper_2310_05205_amd import gear
from tests.helpers import cuda, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_example_runs(bits, dtype):
    from examples import replay_cloning
    say("examples/replay_cloning.py %d bits %s" % (bits, dtype))
    seen = replay_cloning.train(steps=6, windows=16, length=16, bits=bits, dtype=dtype, log=say)
    assert len(seen) == 6 and all(math.isfinite(l) and math.isfinite(n) and n > 0 for l, n in seen)
    assert len(set(seen)) == 6


def test_gradients_of_the_whole_model():
    """Every parameter's gradient in fp32 against the same model in float64 autograd on the CPU."""
    from examples import replay_cloning as example
    torch.manual_seed(3)
    model = example.Cloner().cuda()
    g = torch.Generator().manual_seed(1)
    tokens = torch.randint(0, example.TOKENS, (5, 12), generator=g)
    mask = (torch.rand(5, 12, generator=g) < 0.8).to(torch.uint8)
    weight = 0.5 + torch.rand(5, generator=g)
    say("examples/replay_cloning.py gradients")
    loss, logp = model.loss(tokens.int().to(cuda()), mask.to(cuda()), weight.to(cuda()))
    loss.backward()
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in model.named_parameters()}

    def norm(x, wb):
        c = x - x.mean(-1, keepdim=True)
        return c / torch.sqrt(c.square().mean(-1, keepdim=True) + 1e-5) * wb[0] + wb[1]
    x = p["embed"][tokens[:, :-1]]
    q = norm(x, p["norm"][0]) @ p["project.weight"].t() + p["project.bias"]
    W, h, hs = example.WIDTH, 0.0, []
    for t in range(x.shape[1]):
        f = torch.sigmoid(q[:, t, :W])
        h = f * h + (1 - f) * q[:, t, W:]
        hs.append(h)
    y = norm(torch.stack(hs, 1) + x, p["norm"][1])
    z = torch.log_softmax(y @ p["head"].t(), -1).gather(-1, tokens[:, 1:, None])[..., 0]
    on = mask[:, 1:].double()
    want = -(weight[:, None].double() * on * z).sum() / on.sum()
    want.backward()
    assert abs(float(loss.detach()) - float(want.detach())) < 1e-5 * abs(float(want.detach()))
    for k, v in model.named_parameters():
        # fp32 through some 15 operations, sums of up to 500 terms among them: 2^-24 times a few hundred of the largest gradient.
        off = (v.grad.cpu().double() - p[k].grad).abs().max().item()
        assert off < 400 * 2.0 ** -24 * p[k].grad.abs().max().item(), (k, off)


@pytest.mark.parametrize("bits", [8, 32])
def test_captured_training_steps_replay(bits):
    """A step of norm, token loss, both gradients, clipping and update in one graph, against the same steps run eagerly."""
    n, D, V = 96, 72, 300
    gen = torch.Generator().manual_seed(5)

    def make():
        g = torch.Generator().manual_seed(4)
        bf = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).to(cuda())  # noqa: E731
        p = [bf(V, D), torch.ones(D, device=cuda()), torch.zeros(D, device=cuda())]
        s = {"p": p, "x": bf(n, D), "t": torch.randint(0, V, (n,), generator=g).to(cuda()),
             "master": [p[0].float(), None, None], "step": torch.zeros(1, dtype=torch.int64, device=cuda())}
        kind = torch.float8_e4m3fn if bits == 8 else torch.float32
        s["avg"] = [[torch.zeros(q.numel(), dtype=torch.uint8, device=cuda()).view(kind) if bits == 8 else torch.zeros_like(q, dtype=kind)
                     for q in p] for _ in range(2)]
        s["scales"] = tuple([torch.zeros((q.numel() + 255) // 256, device=cuda()) for q in p] for _ in range(2)) if bits == 8 else None
        return s

    def step(s):
        head, w, b = s["p"]
        y, _, saved = gear.layer_norm(s["x"], w, b, save=True)
        loss, logp, lse = gear.token_loss(y, head, s["t"])
        dy, dhead = gear.token_loss_backward(y, head, s["t"], lse)
        dx, dw, db = gear.layer_norm_backward(dy, s["x"], saved, w)
        grads = [dhead, dw, db]
        norm, factor = gear.grad_norm(grads, max_norm=0.5)
        gear.adamw(s["p"], grads, s["avg"][0], s["avg"][1], s["step"], lr=1e-2, scales=s["scales"], master=s["master"], factor=factor)
        return loss, norm, dx

    def tensors(s):
        return s["p"] + [s["master"][0], s["step"]] + s["avg"][0] + s["avg"][1] + ([] if bits == 32 else s["scales"][0] + s["scales"][1])
    a, b = make(), make()
    say("captured training steps, %d bits" % bits)
    step(a), step(b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(a)
    for _ in range(4):
        x, t = torch.randn(n, D, generator=gen), torch.randint(0, V, (n,), generator=gen)
        for s in (a, b):
            s["x"].copy_(x), s["t"].copy_(t)
        want = step(b)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(got, want))
        assert all(torch.equal(u.view(torch.uint8), v.view(torch.uint8)) for u, v in zip(tensors(a), tensors(b)))
    assert int(a["step"]) == 5
