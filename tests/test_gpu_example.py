"""The example that scores rollouts over an 8-bit cache, against the same decoder
over the 64-bit reference of that cache, rollout by rollout."""
import numpy as np
import pytest

from tests import kv8_reference as R

pytestmark = pytest.mark.gpu


def reference(cfg, rollouts, weights, fmt, beta):
    """Log probabilities, entropies and the LM head's gradient of the example's loss: the rollouts one after the other, in
    the example's pieces and with its bf16 rounding points, K and V through the reference cache, logits in fp32, the
    gradient by autograd."""
    import torch
    m = cfg["model"]
    w = {n: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda().view(torch.bfloat16).float() for n, a in weights.items()}
    w["lm_head"].requires_grad_(True)
    hq, hkv, hd, L = m["n_heads"], m["n_kv_heads"], m["head_dim"], m["n_layers"]
    inv = m["rope_theta"] ** (-torch.arange(0, hd, 2, device="cuda").double() / hd)

    def b(x):
        return x.bfloat16().float()

    def norm(x):
        return b(x * torch.rsqrt((x * x).mean(-1, keepdim=True) + m["rms_eps"]))

    def rope(x, pos):
        a = pos.double()[:, None, None] * inv
        c, s = torch.cos(a).float(), torch.sin(a).float()
        x1, x2 = x.chunk(2, -1)
        return b(torch.cat([x1 * c - x2 * s, x2 * c + x1 * s], -1))

    total, lps, ents, n_tok = 0.0, [], [], sum(len(g) for _, _, g, _ in rollouts)
    for _, prompt, gen, adv in rollouts:
        P, shared = len(prompt), (len(prompt) - 1) // 16 * 16
        n_pages = -(-(P + len(gen)) // 16)
        table = list(range(n_pages))
        caches = [[R.Cache(n_pages, hkv, hd, fmt) for _ in range(2)] for _ in range(L)]
        seq = np.concatenate([prompt, gen])
        cuts = sorted({0, shared} | set(range(P, P + len(gen))))
        hidden = []
        for lo, hi in zip(cuts[:-1], cuts[1:]):
            T, pos = hi - lo, torch.arange(lo, hi, device="cuda")
            h = w["embed"][torch.from_numpy(seq[lo:hi]).long().cuda()]
            for l in range(L):
                x = norm(h)
                q, k = rope(b(x @ w[f"l{l}.wq"].T).view(T, hq, hd), pos), rope(b(x @ w[f"l{l}.wk"].T).view(T, hkv, hd), pos)
                kv = []
                for c, y in zip(caches[l], (k, b(x @ w[f"l{l}.wv"].T).view(T, hkv, hd))):
                    c.write(y.double().cpu().numpy(), table, lo)
                    kv.append(c.read(table, 0, hi))
                o = R.attention(q.double().cpu().numpy(), *kv, np.ones(hi, bool), hi, hd ** -0.5)
                h = h + b(b(torch.from_numpy(o).cuda().float()).view(T, hq * hd) @ w[f"l{l}.wo"].T)
                x = norm(h)
                g = b(torch.nn.functional.silu(b(x @ w[f"l{l}.wg"].T)) * b(x @ w[f"l{l}.wu"].T))
                h = h + b(g @ w[f"l{l}.wd"].T)
            if hi >= P:
                hidden.append(norm(h)[-1:])
        logits = torch.cat(hidden).detach()[:len(gen)] @ w["lm_head"].T
        lp = torch.log_softmax(logits, -1)
        ent = -(lp.exp() * lp).sum(-1)
        got = lp.gather(1, torch.from_numpy(gen).long().cuda()[:, None])[:, 0]
        total = total - (adv * got + beta * ent).sum() / n_tok
        lps.append(got.detach().cpu().numpy())
        ents.append(ent.detach().cpu().numpy())
    total.backward()
    return lps, ents, w["lm_head"].grad


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_scores_match_the_reference_cache(fmt):
    """Both sides round at the same points, so logits differ as two bf16 engines' do: by at most 3e-2 of their rms at two
    layers (the bound of the decoder's own 2-layer tests), a log probability or entropy by twice that, and by the bf16
    rounding of the example's logits (2^-8 of the largest, about 5 rms).  Gradients are linear in the probabilities: within
    10% of their norm."""
    import torch

    import workloads as W
    from examples import score_rollouts as S
    cfg = S.small_config(layers=2, vocab=4096)
    weights, pool = W.make_weights(cfg), W.make_pool(cfg, 0)
    rollouts = S.generate(cfg, pool, weights)[4:14]           # of two prompts at least
    assert len(rollouts) == 10 and len({u for u, _, _, _ in rollouts}) >= 2
    out = S.score(cfg, rollouts, weights, fmt, beta=0.05)
    lps, ents, grad = reference(cfg, rollouts, weights, fmt, 0.05)
    rms = 0.02 * cfg["model"]["d_model"] ** 0.5               # of the logits: unit-rms hidden states, weights of 0.02
    bound = 2 * 3e-2 * rms + 2.0 ** -8 * 5 * rms
    for i, (lp, ent) in enumerate(zip(lps, ents)):
        assert np.max(np.abs(out["logp"][i, :len(lp)] - lp)) <= bound
        assert np.max(np.abs(out["entropy"][i, :len(ent)] - ent)) <= bound
        assert np.all(out["logp"][i, len(lp):] == 0)
    assert float((out["grad"] - grad).norm() / grad.norm()) <= 0.1
    assert torch.isfinite(out["grad"]).all()
