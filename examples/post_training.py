"""One post-training program on the experience path, end to end on one GPU.

A toy policy (a bilinear next-token model with a two-expert head) writes
responses to prompts; a response is rewarded for the share of its tokens below
a limit.  Each iteration goes the way of a GRPO learner:

  responses -> edp_grpo_pack_deliver      (advantages, packed batch)
            -> edp_token_logprob          (log-probabilities under the old policy)
            -> edp_policy_loss_logits     (loss and gradient of the logits)
            -> edp_balance_loss           (the router's term)
            -> weights

and then pairs the best with the worst response of each prompt for one
iteration of preference optimisation:

            -> edp_token_logprob, edp_preference_loss, edp_token_logprob_grad

Matrix products and the optimiser are torch's; every loss and its gradient are
the library's.

    python examples/post_training.py [iterations]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_24456_gb300 import edp  # noqa: E402

VOCAB, DIM, EXPERTS, PROMPTS, GROUP, LENGTH, LIMIT = 515, 64, 8, 24, 8, 40, 64


class Policy:
    """logits[t] = W (E[token t] + the mixture of the token's two best experts)."""

    def __init__(self, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def make(*shape, scale):
            return scale * torch.randn(shape, generator=g, device="cuda")

        self.embed = make(VOCAB, DIM, scale=1.0)
        self.router = make(DIM, EXPERTS, scale=0.3)
        self.experts = make(EXPERTS, DIM, scale=0.1)
        self.head = make(DIM, VOCAB, scale=0.05)
        self.gen = g

    def hidden(self, tokens):
        x = self.embed[tokens.long()]
        scores = x @ self.router
        sel = torch.topk(scores, 2, dim=1)[1].to(torch.int32).contiguous()
        mix = torch.softmax(scores.gather(1, sel.long()), 1)
        return x + (mix[:, :, None] * self.experts[sel.long()]).sum(1), x, scores, sel

    def logits(self, h):
        return (h @ self.head).to(torch.bfloat16)

    def write(self, prompts):
        """A response of LENGTH tokens to each prompt token."""
        out = [prompts]
        for _ in range(LENGTH):
            z = self.logits(self.hidden(out[-1])[0]).float()
            p = torch.softmax(torch.nan_to_num(z).clamp(-50, 50), 1)
            out.append(torch.multinomial(p, 1, generator=self.gen)[:, 0].to(torch.int32))
        return torch.stack(out, 1)


def rows_of(tokens, off):
    """Each row predicts the token after it; a sequence's last row predicts none."""
    target = torch.roll(tokens, -1)
    mask = torch.ones_like(tokens, dtype=torch.uint8)
    mask[off[1:] - 1] = 0
    return target, mask


def train(iterations=40, seed=0, log=print):
    ring = edp.Ring(edp.make_config(16, (1, 4, 4), edp.EDP_XFORM_CHW_NORM_BF16), action=False,
                    reward=False, done=False)
    ctx, policy = ring.ctx, Policy(seed)
    n, room = PROMPTS * GROUP, PROMPTS * GROUP * (LENGTH + 1)
    f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    prompts = torch.arange(PROMPTS, device="cuda", dtype=torch.int32).repeat_interleave(GROUP) + 20
    goff = torch.arange(0, n + 1, GROUP, device="cuda")
    seq_off = torch.arange(0, n + 1, device="cuda") * (LENGTH + 1)
    tokens, value = torch.zeros(room, dtype=torch.int32, device="cuda"), f(room)
    off, adv = torch.zeros(n + 1, dtype=torch.int64, device="cuda"), f(n)
    loss, logp, old, ref = f(8), f(room), f(room), f(room)
    balance, counts = f(1), torch.zeros(EXPERTS, dtype=torch.int64, device="cuda")
    cfg = edp.make_policy_config(0.2, 0.28, dual_clip=3.0, kl_coef=0.001, entropy_coef=0.001,
                                 reduce=edp.EDP_REDUCE_SEQ_MEAN)
    history = dict(reward=[], loss=[], balance=[], preference=[])
    first = None
    for it in range(iterations):
        written = policy.write(prompts)
        reward = (written[:, 1:] < LIMIT).float().mean(1).contiguous()
        order = torch.randperm(n, generator=policy.gen, device="cuda")
        edp.edp_grpo_pack_deliver(ctx, reward, goff, PROMPTS, 1e-6, adv, written.reshape(-1),
                                  seq_off, n, order, n, tokens, off, room, out_value=value)
        target, mask = rows_of(tokens, off)
        for step in range(2):  # two updates per batch: the second is off its policy
            h, x, scores, sel = policy.hidden(tokens)
            z = policy.logits(h)
            if step == 0:
                edp.edp_token_logprob(ctx, z, target, old, mask=mask)
                if first is None:
                    first = policy.head.clone()
                edp.edp_token_logprob(ctx, (h @ first).to(torch.bfloat16), target, ref, mask=mask)
            # the gradient takes the logits' place
            edp.edp_policy_loss_logits(ctx, cfg, z, target, old, value, loss, logp, z,
                                       ref_logp=ref, mask=mask, off=off, n_seq=n)
            dscores = torch.empty_like(scores)
            edp.edp_balance_loss(ctx, scores, sel, 0.1, balance, counts, mask=mask,
                                 dlogits=dscores)
            policy.head -= 40.0 * (h.t() @ z.float())
            policy.router -= 0.5 * (x.t() @ dscores)
        history["reward"].append(float(reward.mean()))
        history["loss"].append(float(loss[0]))
        history["balance"].append(float(balance))
    # the best response of each prompt against its worst
    by_prompt = reward.view(PROMPTS, GROUP)
    place = torch.empty_like(order)
    place[order] = torch.arange(n, device="cuda")  # where a response lies in the packed batch
    start = torch.arange(PROMPTS, device="cuda") * GROUP
    pair = torch.stack([place[start + by_prompt.argmax(1)], place[start + by_prompt.argmin(1)]],
                       1).contiguous()
    h = policy.hidden(tokens)[0]
    z = policy.logits(h)
    stats, dlogp, out = f(room, 2), f(room), f(4)
    edp.edp_token_logprob(ctx, z, target, logp, mask=mask, stats=stats)
    ref.copy_(logp)  # the policy as it is now
    pcfg = edp.make_preference_config(0.5)
    for _ in range(3):
        edp.edp_preference_loss(ctx, pcfg, logp, off, n, room, pair, PROMPTS, out, ref_logp=ref,
                                mask=mask, dlogp=dlogp)
        history["preference"].append(float(out[0]))
        edp.edp_token_logprob_grad(ctx, z, target, stats, dlogp, z, mask=mask)
        policy.head -= 0.005 * (h.t() @ z.float())
        z = policy.logits(h)
        edp.edp_token_logprob(ctx, z, target, logp, mask=mask, stats=stats)
    edp.edp_sync(ctx)
    ring.close()
    log("reward %.3f -> %.3f, balance %.4f -> %.4f, preference loss %s" % (
        history["reward"][0], history["reward"][-1], history["balance"][0],
        history["balance"][-1], " -> ".join("%.4f" % x for x in history["preference"])))
    return history


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 40)
