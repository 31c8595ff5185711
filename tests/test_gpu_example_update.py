"""The example's update: attention over shared prompts and the loss through the
LM head, as they are used together."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_the_update(fmt):
    """Grouped and plain attention round to bf16 alike, so logits differ as two bf16 engines' do: by at most 3e-2 of their rms
    at two layers.  From the hidden states on the loss is fp32 against 64 bits: log probabilities and entropies by
    d 2^-24 sum |h w| and 2^-18 (1 + |.|); gradients by what their bf16 parts leave (2^-8 of |D| times the other side for
    the hidden states', which are rounded once more; 2^-16 for the LM head's) beside twice that log probability's error
    of every element of D."""
    import torch

    import workloads as W
    from examples import score_rollouts as S
    cfg = S.small_config(layers=2, vocab=4096)
    weights, pool = W.make_weights(cfg), W.make_pool(cfg, 0)
    rollouts = [r for r in S.generate(cfg, pool, weights)[4:14] if len(r[2])]
    assert len({u for u, _, _, _ in rollouts}) >= 2
    beta = 0.05
    out = S.update(cfg, rollouts, weights, fmt, beta)
    plain = S.update(cfg, rollouts, weights, fmt, beta, grouped=False)
    head = S.upload(weights)["lm_head"].double()
    h, tok = out["hidden"].double(), out["tok"].long()[:, None]
    logits = h @ head.T.contiguous()
    other = plain["hidden"].double() @ head.T.contiguous()
    assert float((logits - other).pow(2).mean().sqrt()) <= 3e-2 * float(logits.pow(2).mean().sqrt())

    lp = torch.log_softmax(logits, -1)
    p = lp.exp()
    logp, ent = lp.gather(1, tok)[:, 0], -(p * lp).sum(-1)
    moved = 2 * (h.shape[1] + 4) * 2.0 ** -24 * (h.abs() @ head.abs().T.contiguous()).amax(-1)
    assert bool(((out["logp"] - logp).abs() <= moved + 2.0 ** -18 * (1 + logp.abs())).all())
    assert bool(((out["entropy"] - ent).abs() <= 2 * moved * (1 + ent) + 2.0 ** -18 * (1 + ent)).all())
    g, ge = out["g"].double()[:, None], -beta / len(tok)
    D = -p * (g + ge * (lp + ent[:, None]))
    D.scatter_add_(1, tok, g)
    Derr = (moved[:, None] + 2.0 ** -17) * p * (g.abs() + abs(ge) * (lp.abs() + ent[:, None] + 2)) + 2.0 ** -22 * D.abs()
    for got, A, E, B, part in ((out["grad_hidden"], D, Derr, head, 2.0 ** -8),
                               (out["grad"], D.T.contiguous(), Derr.T.contiguous(), h, 2.0 ** -16)):
        want = A @ B
        bound = E @ B.abs() + (part + (A.shape[1] + 8) * 2.0 ** -24) * (A.abs() @ B.abs())
        bound = bound + torch.finfo(got.dtype).eps / 2 * (want.abs() + bound)
        assert bool(((got.double() - want).abs() <= bound).all())
