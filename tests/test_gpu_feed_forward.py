"""The feed-forward block made of the layer operators: its outputs and gradients against the same block in 64 bits
under autograd, and a few steps of training."""
import pytest
import torch

import operators_ref as R
import paper_1801_04928_b200 as lf

pytestmark = pytest.mark.gpu


def _reference(x, p, w1, w2):
    """Block in 64 bits with the 16-bit weights; p: fp32 parameters."""
    h = x / (x.square().mean(1, keepdim=True) + 1e-5).sqrt() * p["gain"]
    return R.act(h @ w1.t() + p["b1"], R.GELU) @ w2.t() + p["b2"] + x


@pytest.mark.parametrize("tokens,width,hidden", [(3, 64, 256), (130, 264, 520), (700, 512, 2048)])
def test_block_against_autograd(tokens, width, hidden):
    from paper_1801_04928_b200.feed_forward import FeedForwardBlock
    g = torch.Generator(device="cuda")
    g.manual_seed(tokens)
    with lf.Operators(lf.lf_ops_workspace(tokens, hidden)) as ops:
        block = FeedForwardBlock(ops, tokens, width, hidden, seed=tokens)
        for k in ("b1", "b2", "gain"):
            block.master[k].add_(torch.empty_like(block.master[k]).normal_(0, 0.2, generator=g))
        x = torch.empty(tokens, width, device="cuda").normal_(0, 1, generator=g).to(torch.bfloat16)
        dy = torch.empty(tokens, width, device="cuda").normal_(0, 1, generator=g).to(torch.bfloat16)
        y, dx = torch.empty_like(x), torch.empty_like(x)
        block.forward(x, y)
        block.backward(x, dy, dx)
        ops.sync()
    leaf = {k: v.to(R.D).requires_grad_(True) for k, v in block.master.items() if k not in ("w1", "w2")}
    leaf["w1"], leaf["w2"], leaf["x"] = (t.to(R.D).requires_grad_(True) for t in (block.w1, block.w2, x))
    ref = _reference(leaf["x"], leaf, leaf["w1"], leaf["w2"])
    ref.backward(dy.to(R.D))
    far = lambda got, want: ((got.to(R.D) - want).norm() / want.norm()).item()   # noqa: E731
    # u, a and y are rounded to bf16 once each on the way: at most 2^-8 of every value three times over
    assert far(y, ref.detach()) <= 3 * 2.0 ** -8
    # the 8-bit values are at most 2^-4 off (and a rounding to 16 bits); gelu is 1.13-Lipschitz and gelu'' <= 1.2 / sigma
    # of |z| about 1, so that nothing is off by more than 1.2 * 2^-4 plus the 16-bit roundings
    bound = 1.2 * 2.0 ** -4 + 4 * 2.0 ** -8
    for k, got in block.grad.items():
        assert far(got, leaf[k].grad) <= bound, k
    assert far(dx, leaf["x"].grad) <= bound


def test_training_lowers_the_loss():
    from paper_1801_04928_b200.feed_forward import train
    losses, block, ops, x = train(512, 128, 512, 25)
    assert losses[-1] < 0.6 * losses[0] and all(b < a for a, b in zip(losses, losses[1:])), losses
    # one token through the few-token kernels gives what it gave among the others, up to bf16 roundings
    y, one = torch.empty_like(x), torch.empty_like(x[:1])
    block.forward(x, y, keep=False)
    block.forward(x[5:6], one, keep=False)
    ops.sync()
    d = (one[0].double() - y[5].double()).norm() / y[5].double().norm()
    assert d.item() <= 2 * 2.0 ** -8
    ops.close()
