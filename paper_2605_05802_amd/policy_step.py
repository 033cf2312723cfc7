"""One GRPO step from rollout to update, on a small random decoder (prints a line per update).

The library rolls out groups of sampled trajectories, scores nothing twice: the logits that each sampled token came from are
kept.  A small adapter on top of them is then trained -- logits + dropout(norm(A[previous token])) B + c, with A, B, c and the norm's
gain the trained tensors, norm and dropout where they are asked for -- so that the whole way from tokens to updated weights is here
without a training stack:

    sr_embed, sr_add_norm, sr_dropout    the adapter's rows, and sr_embed_grad, sr_add_norm_grad, sr_dropout their gradients
    sr_grpo_loss        advantages of the groups' rewards (Eq. 1)
    sr_policy_loss      log-probabilities of the rollout (the loss alone), then loss and gradient of the logits per update
    sr_preference_loss  the best against the worst member of every group whose rewards differ
    sr_clip_grad_norm   the adapter's gradients, which torch multiplies out of the logits', scaled down to a largest norm

    python -m paper_2605_05802_amd.policy_step [--norm] [--dropout 0.1]
"""
from __future__ import annotations

import argparse
from types import SimpleNamespace

import torch

from . import (GRAD_NORM_WORKSPACE, Context, Dropout, embed_grad_workspace, norm_grad_workspace, sr_add_norm, sr_add_norm_grad, sr_clip_grad_norm,
               sr_dropout, sr_embed, sr_embed_grad, sr_grpo_loss, sr_policy_loss, sr_preference_loss, tensor_list, token_loss_workspace)

SHAPE = SimpleNamespace(n_layers=2, hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn=688, vocab=1024, rms_eps=1e-6,
                        rope_theta=1e6, qkv_bias=True)


def random_weights(ctx: Context, s, gen):
    mat = lambda *shape: (0.02 * torch.randn(*shape, generator=gen, device="cuda")).bfloat16()
    ones = lambda: torch.ones(s.hidden, dtype=torch.bfloat16, device="cuda")
    q, kv = s.n_q_heads * s.head_dim, s.n_kv_heads * s.head_dim
    layers = [dict(wq=mat(q, s.hidden), wk=mat(kv, s.hidden), wv=mat(kv, s.hidden), wo=mat(s.hidden, q), wg=mat(s.ffn, s.hidden),
                   wu=mat(s.ffn, s.hidden), wd=mat(s.hidden, s.ffn), bq=mat(q), bk=mat(kv), bv=mat(kv), norm1=ones(), norm2=ones())
              for _ in range(s.n_layers)]
    ctx.sr_load_weights(mat(s.vocab, s.hidden), mat(s.vocab, s.hidden), ones(), layers)


def rollout(groups: int, G: int, turns: int, obs_len: int, act_len: int, seed: int):
    """Sampled trajectories: tokens, the tokens before them, and the logits they were drawn from, trajectory by trajectory."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    prompt_len, n = 32, groups * G
    ctx = Context(SHAPE, groups, G, 0.3, page_tokens=32, max_seq_len=prompt_len + turns * (obs_len + act_len), max_turns=turns,
                  kv_pool_bytes=1 << 27, temperature=1.0, sample_seed=seed)
    random_weights(ctx, SHAPE, gen)
    ids = lambda *shape: torch.randint(0, SHAPE.vocab, shape, generator=gen, device="cuda", dtype=torch.int32)
    ctx.sr_prefill_chunk(ids(groups, prompt_len), True)
    logits = torch.empty(n, turns * act_len, SHAPE.vocab, device="cuda")
    tokens = torch.empty(n, turns * act_len, dtype=torch.int32, device="cuda")
    before = torch.empty_like(tokens)
    now, step = torch.empty(n, SHAPE.vocab, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    for turn in range(turns):
        obs = ids(n, obs_len)
        ctx.sr_prefill_chunk(obs, False)
        last = obs[:, -1]
        for a in range(act_len):
            at = turn * act_len + a
            ctx.sr_get_logits(now)
            ctx.sr_decode_step(None, step)
            logits[:, at], tokens[:, at], before[:, at] = now, step, last
            last = tokens[:, at]
    ctx.close()
    return logits.view(-1, SHAPE.vocab), tokens.view(-1), before.view(-1).long()


class Adapter:
    """logits + dropout(norm(A[previous token])) B + c"""

    def __init__(self, rank: int, seed: int, dropout: float = 0.0, norm: bool = False):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.A = torch.randn(SHAPE.vocab, rank, generator=gen, device="cuda") / rank ** 0.5
        self.B = torch.zeros(rank, SHAPE.vocab, device="cuda")
        self.c = torch.zeros(SHAPE.vocab, device="cuda")
        self.gain = torch.ones(rank, device="cuda") if norm else None
        self.weights = (self.A, self.B, self.c) + ((self.gain,) if norm else ())
        self.grads = tuple(torch.zeros_like(w) for w in self.weights)
        self.listed = tensor_list(self.grads)                  # the plan of the norm: the gradients stay where they are
        self.norm = torch.empty(1, device="cuda")
        self.workspace = torch.empty(GRAD_NORM_WORKSPACE, dtype=torch.uint8, device="cuda")
        # a mask for every update: their number lies on the device
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.dropout = Dropout(dropout, seed, step=self.step) if dropout else None

    def rows(self, before):
        """(tokens, rows of A, rstd of the norm, what is multiplied by B)"""
        new = lambda *shape: torch.empty(*shape, device="cuda")
        tokens, (n, rank) = before.int(), (len(before), self.A.shape[1])
        rows, rstd = new(n, rank), None
        sr_embed(self.A, tokens, rows)
        fed = rows
        if self.gain is not None:
            fed, rstd = new(n, rank), new(n)
            sr_add_norm(rows, self.gain, fed, rstd=rstd)
        if self.dropout:
            normed, fed = fed, new(n, rank)
            sr_dropout(normed, fed, self.dropout)
        return tokens, rows, rstd, fed

    def logits(self, base, before):
        return base + self.rows(before)[3] @ self.B + self.c

    def gradients(self, d_logits, before):
        """Of the trained tensors, from that of the logits."""
        tokens, rows, rstd, fed = self.rows(before)
        n, rank = rows.shape
        d = d_logits @ self.B.t()
        torch.mm(fed.t(), d_logits, out=self.grads[1])
        torch.sum(d_logits, 0, out=self.grads[2])
        workspace = torch.empty(max(embed_grad_workspace(n, rank), norm_grad_workspace(n, rank)), dtype=torch.uint8, device="cuda")
        if self.dropout:
            sr_dropout(d, d, self.dropout)
        if self.gain is not None:
            sr_add_norm_grad(d, rows, rstd, self.gain, workspace, d_x=d, d_gain=self.grads[3])
        sr_embed_grad(d, tokens, self.grads[0], workspace)
        return self.grads

    def update(self, d_logits, before, rate: float, max_norm: float):
        self.gradients(d_logits, before)
        sr_clip_grad_norm(self.listed, max_norm, self.norm, self.workspace)
        for w, g in zip(self.weights, self.grads):
            w.sub_(rate * g)
        self.step.add_(1)
        return self.norm.item()


def train(groups=8, G=8, turns=3, obs_len=16, act_len=8, updates=6, pair_updates=4, rate=20.0, max_norm=0.1, kl_coef=0.02, seed=0,
          dropout=0.0, norm=False, say=lambda line: None):
    """Returns the losses of the policy updates, those of the preference updates, and the gradient norms."""
    base, tokens, before = rollout(groups, G, turns, obs_len, act_len, seed)
    n, rows, each = groups * G, groups * G * turns * act_len, turns * act_len
    seq_start = torch.arange(0, rows + 1, each, dtype=torch.int32, device="cuda")
    # a reward that the tokens decide: trajectories with more tokens than most from the lower half of the vocabulary
    low = (tokens.view(n, each) < SHAPE.vocab // 2).sum(1)
    rewards = (low > each // 2).float()

    stats, workspace = torch.empty(4, device="cuda"), torch.empty(token_loss_workspace(rows, n), dtype=torch.uint8, device="cuda")
    old, grad = torch.empty(rows, device="cuda"), torch.empty_like(base)
    advantages = torch.zeros(n, device="cuda")
    # the rollout's own log-probabilities: the loss alone, whatever the ratio
    sr_policy_loss(base, tokens, seq_start, torch.zeros_like(old), advantages, stats, workspace, token_logprob=old)
    sr_grpo_loss(old.view(n, each).double().sum(1), rewards, G, 1e-6, advantages, torch.empty(groups, dtype=torch.float64, device="cuda"),
                 torch.empty(1, dtype=torch.float64, device="cuda"))

    adapter, losses, norms = Adapter(16, seed, dropout, norm), [], []
    for u in range(updates):
        sr_policy_loss(adapter.logits(base, before), tokens, seq_start, old, advantages, stats, workspace, ref_logprob=old, grad=grad,
                       kl_coef=kl_coef, reduce="sequences")
        norms.append(adapter.update(grad, before, rate, max_norm))
        loss, surrogate, kl, clipped = stats.tolist()
        losses.append(loss)
        say(f"policy update {u}: loss {loss:+.5f}, surrogate {surrogate:+.5f}, KL {kl:.5f}, clipped {clipped:.3f}, gradient norm {norms[-1]:.4f}")

    # the best and the worst member of every group whose rewards differ
    r = rewards.view(groups, G)
    mixed = (r.max(1).values > r.min(1).values).nonzero()[:, 0]
    pair_losses = []
    if len(mixed):
        members = torch.stack([r.argmax(1), r.argmin(1)], 1)[mixed] + G * mixed[:, None]
        take = (members.reshape(-1)[:, None] * each + torch.arange(each, device="cuda")).reshape(-1)
        chosen, tok, prev, ref = base[take], tokens[take].contiguous(), before[take], old[take].contiguous()
        starts = torch.arange(0, len(take) + 1, each, dtype=torch.int32, device="cuda")
        for u in range(pair_updates):
            logits = adapter.logits(chosen, prev)
            sr_preference_loss(logits, tok, starts, stats, workspace, ref_logprob=ref, grad=logits, beta=0.1)   # in place
            norms.append(adapter.update(logits, prev, rate, max_norm))
            loss, right, better, worse = stats.tolist()
            pair_losses.append(loss)
            say(f"preference update {u}: loss {loss:.5f}, pairs in order {right:.2f}, rewards {better:+.4f} and {worse:+.4f}, "
                f"gradient norm {norms[-1]:.4f}")
    return losses, pair_losses, norms


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--groups", type=int, default=8)
    ap.add_argument("--G", type=int, default=8)
    ap.add_argument("--updates", type=int, default=6)
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--dropout", type=float, default=0.0, help="of the adapter's rows")
    ap.add_argument("--norm", action="store_true", help="norm the adapter's rows")
    args = ap.parse_args()
    assert torch.cuda.is_available(), "needs a GPU"
    train(groups=args.groups, G=args.G, updates=args.updates, seed=args.seed, dropout=args.dropout, norm=args.norm, say=print)


if __name__ == "__main__":
    main()
