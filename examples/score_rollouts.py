"""Score the rollouts of one allocation step over an 8-bit KV cache and form
the policy gradient of their tokens.

    python examples/score_rollouts.py [--format int8|fp8] [--layers N]

1. An allocation step of the 1.5B-shaped workload (cut to a few layers and
   prompts) generates rollouts; sara_finish_step gives their advantages.
2. The committed rollouts go through the same decoder again, written in torch
   over a paged 8-bit cache: sara_kv8_write and sara_kv8_attention in every
   layer.  Whole pages of a prompt are written once and shared by its rollouts;
   the rest of the prompt is one ragged piece a rollout, and the generated
   tokens follow one by one, as a server would take them.
3. sara_token_logprobs gives each token's log probability, the entropy and the
   most likely alternatives; sara_token_logprobs_grad the gradient of
   -sum(advantage * log p + beta * entropy) / tokens with respect to the logits,
   from which the LM head's gradient is accumulated.
4. The same loss as an update takes it: each answer is one ragged piece, whose
   attention takes the prompt's pages as its group's (sara_kv8_group_attention),
   and all tokens together go through the LM head without logits in memory
   (sara_head_logprobs, sara_head_logprobs_grad), which give the gradients of the
   LM head and of the hidden states.
"""
import argparse
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_26253_amd as sara  # noqa: E402
import workloads as W  # noqa: E402

PAGE = 16


class CachedDecoder:
    """The workloads' decoder (bf16 weights) in torch, its K and V in 8-bit pages."""

    def __init__(self, model, weights, n_pages, fmt):
        self.m, self.w = model, weights
        hkv, hd = model["n_kv_heads"], model["head_dim"]
        dt = torch.int8 if fmt == "int8" else torch.float8_e4m3fn

        def pages():
            return torch.zeros((n_pages, hkv, PAGE, hd), dtype=torch.uint8, device="cuda").view(dt)

        def exponents():
            return torch.zeros((n_pages, hkv), dtype=torch.uint8, device="cuda")

        self.cache = [(pages(), pages(), exponents(), exponents()) for _ in range(model["n_layers"])]
        self.inv_freq = model["rope_theta"] ** (-torch.arange(0, hd, 2, device="cuda", dtype=torch.float64) / hd)

    def norm(self, x, gain):
        return (x * torch.rsqrt((x * x).mean(-1, keepdim=True) + self.m["rms_eps"]) * gain.float()).bfloat16()

    def rope(self, x, pos):
        a = pos.double()[:, None, None] * self.inv_freq
        c, s = torch.cos(a).float(), torch.sin(a).float()
        x1, x2 = x.float().chunk(2, -1)
        return torch.cat([x1 * c - x2 * s, x2 * c + x1 * s], -1).bfloat16()

    def forward(self, tokens, pos, table, start, off, ctx, max_ctx, groups=None):
        """Hidden states of new tokens: rows off[i]..off[i + 1] (one a sequence without `off`) follow the start[i] tokens
        that the cache holds of sequence i; ctx[i] counts both.  groups: (first sequences, tokens in common, most of them)
        of sequences that share a prompt's pages."""
        m, w = self.m, self.w
        hq, hkv, hd, T = m["n_heads"], m["n_kv_heads"], m["head_dim"], len(tokens)
        h = w["embed"][tokens.long()].float()
        for l, cache in enumerate(self.cache):
            x = self.norm(h, w[f"l{l}.attn_norm"])
            q = self.rope((x @ w[f"l{l}.wq"].T).view(T, hq, hd), pos)
            k = self.rope((x @ w[f"l{l}.wk"].T).view(T, hkv, hd), pos)
            v = (x @ w[f"l{l}.wv"].T).view(T, hkv, hd)
            sara.sara_kv8_write(*cache, k, v, table, start, off)
            o = torch.empty_like(q)
            if groups is None:
                sara.sara_kv8_attention(q, *cache, table, ctx, off, o, max_ctx=max_ctx)
            else:
                sara.sara_kv8_group_attention(q, *cache, table, ctx, off, groups[0], groups[1], o, max_ctx=max_ctx, max_shared=groups[2])
            h = h + (o.view(T, hq * hd) @ w[f"l{l}.wo"].T).float()
            x = self.norm(h, w[f"l{l}.ffn_norm"])
            g = torch.nn.functional.silu((x @ w[f"l{l}.wg"].T).float()) * (x @ w[f"l{l}.wu"].T).float()
            h = h + (g.bfloat16() @ w[f"l{l}.wd"].T).float()
        return self.norm(h, w["final_norm"])


def i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


def generate(cfg, pool, weights):
    """Rollouts of one allocation step: (prompt, generated tokens, advantage) of each committed rollout, and the prompt it
    belongs to."""
    specs = W.weight_specs(cfg["model"])
    ctx = sara.Sara(cfg["model"], cfg["alloc"], W.sampling_seed(cfg), sara.upload_weights(specs, weights))
    ctx.sara_begin_step(i32(pool["tokens"]), pool["offsets"], torch.from_numpy(pool["p"]).cuda(), None, 0)
    ctx.sara_run()
    ctx.sara_finish_step(1e-6)
    roll = ctx.read_rollouts()
    off, _, adv = ctx.read_advantages()
    k, out = cfg["alloc"]["k"], []
    for g, u in enumerate(np.flatnonzero(roll["status"] == sara.SARA_COMMITTED)):
        prompt = pool["tokens"][pool["offsets"][u]:pool["offsets"][u + 1]]
        for j in range(off[g + 1] - off[g]):
            r = u * k + j
            out.append((int(u), prompt, roll["tokens"][r, :roll["length"][r]], float(adv[off[g] + j])))
    ctx.close()
    return out


def upload(weights):
    return {n: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda().view(torch.bfloat16) for n, a in weights.items()}


def lay_out(rollouts):
    """Lengths of prompts and answers, tokens in whole pages of a prompt (its last token apart), page tables in which a
    prompt's rollouts have those in common, the first rollout of each prompt, and the pages of them all."""
    plen = np.array([len(p) for _, p, _, _ in rollouts])
    glen = np.array([len(g) for _, _, g, _ in rollouts])
    shared = (plen - 1) // PAGE * PAGE
    width = int(-(-(plen + glen).max() // PAGE))
    table, at, of_prompt = np.full((len(rollouts), width), -1, np.int64), 0, {}
    for i, (u, _, _, _) in enumerate(rollouts):
        common = shared[i] // PAGE
        if u not in of_prompt:
            of_prompt[u] = (i, np.arange(at, at + common))
            at += common
        own = -(-(plen[i] + glen[i]) // PAGE) - common
        table[i, :common], table[i, common:common + own] = of_prompt[u][1], np.arange(at, at + own)
        at += own
    return plen, glen, shared, table, [i for i, _ in of_prompt.values()], at


def score(cfg, rollouts, weights, fmt="int8", beta=0.01, n_top=3):
    """Log probabilities, entropies and alternatives of the rollouts' tokens, and the gradient of the LM head."""
    w = upload(weights)
    n = len(rollouts)
    plen, glen, shared, table, of_prompt, at = lay_out(rollouts)
    max_ctx = table.shape[1] * PAGE
    dec = CachedDecoder(cfg["model"], w, max(at, 1), fmt)
    tab = i32(table)
    weight = 1.0 / int(glen.sum())
    adv = torch.tensor([a for _, _, _, a in rollouts], device="cuda", dtype=torch.float32)
    out = dict(logp=np.zeros((n, int(glen.max()))), entropy=np.zeros((n, int(glen.max()))),
               top=np.full((n, int(glen.max()), n_top), -1), grad=torch.zeros(w["lm_head"].shape, device="cuda"))

    def piece(seqs, starts, tokens):
        """New tokens of the rollouts `seqs`: their hidden states."""
        lens = [len(t) for t in tokens]
        off = np.concatenate([[0], np.cumsum(lens)])
        pos = np.concatenate([s + np.arange(c) for s, c in zip(starts, lens)])
        return dec.forward(i32(np.concatenate(tokens)), i32(pos), tab[i32(seqs).long()].contiguous(), i32(starts),
                           None if max(lens) == 1 else i32(off), i32(np.asarray(starts) + lens), max_ctx), off

    def take(seqs, hidden, i):
        """Token i of the rollouts `seqs` under the hidden states before it."""
        r = len(seqs)
        tok, idx = i32([rollouts[s][2][i] for s in seqs]), i32(seqs).long()
        logits = hidden @ w["lm_head"].T
        logp, ent = torch.empty(r, device="cuda"), torch.empty(r, device="cuda")
        stats = torch.empty((r, 2), device="cuda")
        ids, lps = torch.empty((r, n_top), device="cuda", dtype=torch.int32), torch.empty((r, n_top), device="cuda")
        sara.sara_token_logprobs(logits, tok, logp, ent, stats, ids, lps)
        g = -weight * adv[idx]
        sara.sara_token_logprobs_grad(logits, tok, stats, ent, g, torch.full_like(g, -weight * beta), logits)   # in place
        out["grad"].addmm_(logits.T.float(), hidden.float())
        out["logp"][seqs, i], out["entropy"][seqs, i] = logp.cpu().numpy(), ent.cpu().numpy()
        out["top"][seqs, i] = ids.cpu().numpy()

    # the prompts' whole pages, once a prompt
    first = [i for i in of_prompt if shared[i]]
    if first:
        piece(first, [0] * len(first), [rollouts[i][1][:shared[i]] for i in first])
    # the rest of each rollout's prompt, in pages of its own
    seqs = np.flatnonzero(glen > 0)
    hidden, off = piece(seqs, shared[seqs], [rollouts[i][1][shared[i]:] for i in seqs])
    take(seqs, hidden[torch.from_numpy(off[1:] - 1).cuda()], 0)
    # the generated tokens, one a rollout and step
    for i in range(1, int(glen.max())):
        seqs = np.flatnonzero(glen > i)
        hidden, _ = piece(seqs, plen[seqs] + i - 1, [rollouts[s][2][i - 1:i] for s in seqs])
        take(seqs, hidden, i)
    return out


def update(cfg, rollouts, weights, fmt="int8", beta=0.01, grouped=True):
    """The loss's log probabilities and entropies of all tokens, one rollout's after the other's, the hidden states before
    them, and the gradients of both sides of the LM head.  A prompt's rollouts follow each other."""
    w = upload(weights)
    plen, glen, shared, table, of_prompt, at = lay_out(rollouts)
    max_ctx, tab = table.shape[1] * PAGE, i32(table)
    dec = CachedDecoder(cfg["model"], w, max(at, 1), fmt)
    first = [i for i in of_prompt if shared[i]]
    if first:
        tokens = [rollouts[i][1][:shared[i]] for i in first]
        off = np.concatenate([[0], np.cumsum([len(t) for t in tokens])])
        dec.forward(i32(np.concatenate(tokens)), i32(np.concatenate([np.arange(len(t)) for t in tokens])), tab[i32(first).long()].contiguous(),
                    i32(np.zeros(len(first))), i32(off), i32(shared[first]), max_ctx)
    # what is left of a prompt and its answer but for the last token
    tokens = [np.concatenate([p[s:], g[:-1]]) for (_, p, g, _), s in zip(rollouts, shared)]
    off = np.concatenate([[0], np.cumsum([len(t) for t in tokens])])
    pos = np.concatenate([s + np.arange(len(t)) for t, s in zip(tokens, shared)])
    groups = (i32(of_prompt + [len(rollouts)]), i32(shared[of_prompt]), int(shared.max())) if grouped else None
    hidden = dec.forward(i32(np.concatenate(tokens)), i32(pos), tab, i32(shared), i32(off), i32(shared + np.diff(off)), max_ctx, groups)
    before = np.concatenate([np.arange(off[i + 1] - g, off[i + 1]) for i, g in enumerate(glen)])
    hidden = hidden[i32(before).long()].contiguous()
    tok = i32(np.concatenate([g for _, _, g, _ in rollouts]))
    adv = np.repeat([a for _, _, _, a in rollouts], glen)
    T = len(tok)
    logp, ent, stats = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty((T, 2), device="cuda")
    sara.sara_head_logprobs(hidden, w["lm_head"], tok, logp, ent, stats)
    g = torch.tensor(-adv / T, device="cuda", dtype=torch.float32)
    grad_hidden, grad = torch.empty_like(hidden), torch.empty(w["lm_head"].shape, device="cuda")
    sara.sara_head_logprobs_grad(hidden, w["lm_head"], tok, stats, ent, g, torch.full_like(g, -beta / T), grad_hidden, grad)
    return dict(logp=logp, entropy=ent, hidden=hidden, tok=tok, g=g, grad_hidden=grad_hidden, grad=grad)


def small_config(layers=2, vocab=None):
    cfg = W.parity_slice(W.get_config("qwen1p5b_shape"), B=4, max_new=24, prompt_len=(20, 90))
    cfg["model"]["n_layers"] = layers
    if vocab:
        cfg["model"].update(vocab=vocab, eos_id=vocab - 1)
    return cfg


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--format", choices=("int8", "fp8"), default="int8")
    ap.add_argument("--layers", type=int, default=2)
    a = ap.parse_args()
    cfg = small_config(a.layers)
    weights, pool = W.make_weights(cfg), W.make_pool(cfg, 0)
    rollouts = generate(cfg, pool, weights)
    if not rollouts:
        print("no group was committed")
        return
    out = score(cfg, rollouts, weights, a.format)
    n_tok = sum(len(g) for _, _, g, _ in rollouts)
    hit = np.mean([out["top"][i, j, 0] == g[j] for i, (_, _, g, _) in enumerate(rollouts) for j in range(len(g))])
    print(f"{len(rollouts)} rollouts, {n_tok} tokens: mean log p {out['logp'].sum() / n_tok:.4f} "
          f"(uniform {-math.log(cfg['model']['vocab']):.4f}), mean entropy {out['entropy'].sum() / n_tok:.4f}, "
          f"most likely id sampled {100 * hit:.1f}%, LM head gradient norm {float(out['grad'].norm()):.4e}")
    out = update(cfg, rollouts, weights, a.format)
    print(f"the update: mean log p {float(out['logp'].mean()):.4f}, mean entropy {float(out['entropy'].mean()):.4f}, "
          f"LM head gradient norm {float(out['grad'].norm()):.4e}, hidden states' {float(out['grad_hidden'].float().norm()):.4e}")


if __name__ == "__main__":
    main()
