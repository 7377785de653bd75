"""Rollouts of a policy, drafted by a copy of its head in 4 bits and verified by the head itself, and a step of the clipped policy loss on them.

The body of the model stands still: a random feature vector for every token, so that the logits of a position are the head's on the
features of the token before it.  In each round the drafter proposes some tokens a request one after another (matvec4, draw_tokens), the head sees all
of their positions at once, and verify_draft keeps what stands: the answers are distributed as if the head had drawn every token, and the
log-probabilities that come with them are what policy_loss takes.

    python examples/speculative_rollouts.py [--vocab 4096] [--width 256] [--requests 16] [--drafts 4] [--tokens 48]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2203_16340_amd as L  # noqa: E402


def roll_out(head, weights, features, first, drafts, tokens, gen):
    """(answers, logp, lengths, rounds): requests x tokens of what was emitted after each `first` token, -1 and 0 behind an answer's end.  head: (vocab, width);
    weights: the same in 4 bits."""
    n, dev = len(first), first.device
    answers = torch.full((n, tokens + drafts + 1), -1, dtype=torch.int64, device=dev)
    logp = torch.zeros(n, tokens + drafts + 1, device=dev)
    length = torch.zeros(n, dtype=torch.int64, device=dev)
    last, rounds = first, 0
    while int(length.min()) < tokens:
        rounds += 1
        seen, proposed, drafter, given = [last], [], [], []
        for _ in range(drafts):
            z = L.matvec4(features[seen[-1]], weights)
            d = L.draw_tokens(z, torch.rand(n, device=dev, generator=gen))
            seen.append(d.tokens)
            proposed.append(d.tokens)
            drafter.append(z)
            given.append(d.logp)
        z = (features[torch.stack(seen, 1)] @ head.t()).contiguous()                  # requests x (drafts + 1) x vocab
        # requests that are done have ended: nothing of theirs is looked at
        lengths = torch.where(length < tokens, drafts, -1)
        r = L.verify_draft(z, torch.stack(proposed, 1), torch.rand(n, drafts, device=dev, generator=gen), torch.rand(n, device=dev, generator=gen),
                           draft_logits=torch.stack(drafter, 1), draft_logp=torch.stack(given, 1), lengths=lengths)
        at = length[:, None] + torch.arange(drafts + 1, device=dev)
        kept = r.tokens >= 0
        rows = torch.arange(n, device=dev)[:, None].expand_as(at)
        answers[rows[kept], at[kept]] = r.tokens[kept]
        logp[rows[kept], at[kept]] = r.logp[kept]
        newest = r.tokens.gather(1, (r.count - 1).clamp(min=0)[:, None])[:, 0]
        last = torch.where(r.count > 0, newest, last)
        length += r.count
    return answers[:, :tokens].contiguous(), logp[:, :tokens].contiguous(), length.clamp(max=tokens), rounds


def positions(features, first, answers):
    """the features that each token of the answers was drawn behind, one row a token"""
    before = torch.cat([first[:, None], answers[:, :-1]], 1)
    return features[before.clamp(min=0)].flatten(0, 1)


def policy_step(head, features, first, answers, logp, value):
    """The clipped policy loss on the answers and its gradient with respect to the head; value: the reward of each token of the vocabulary."""
    x, y = positions(features, first, answers), answers.flatten()
    got = value[y]
    adv = ((got - got.mean()) / got.std()).contiguous()
    z = x @ head.t()
    r = L.policy_loss(z.contiguous(), y, logp.flatten(), adv, weight=torch.full_like(got, 1.0 / len(y)), entropy_coef=1e-3)
    return r, r.grad.t() @ x


def run(vocab=4096, width=256, requests=16, drafts=4, tokens=48, steps=3, lr=8.0, seed=0, device="cuda:0"):
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    features = torch.randn(vocab, width, device=device, generator=gen)
    head = torch.randn(vocab, width, device=device, generator=gen) * (2.5 / width ** 0.5)
    value = torch.randn(vocab, device=device, generator=gen)
    first = torch.randint(0, vocab, (requests,), device=device, generator=gen)
    out = []
    for _ in range(steps):
        group = 128 if width % 128 == 0 else 32
        weights = L.pack4(*L.quantize4(head, group=group), cols=width, group=group)
        answers, logp, length, rounds = roll_out(head, weights, features, first, drafts, tokens, gen)
        r, grad = policy_step(head, features, first, answers, logp, value)
        out.append(dict(answers=answers, logp=logp, length=length, rounds=rounds, loss=r.loss, grad=grad, head=head.clone(), reward=value[answers].mean()))
        head = head - lr * grad
    return dict(features=features, first=first, value=value, steps=out)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("vocab", 4096), ("width", 256), ("requests", 16), ("drafts", 4), ("tokens", 48), ("steps", 3), ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=default)
    args = ap.parse_args()
    for k, s in enumerate(run(**vars(args))["steps"]):
        print(f"step {k}: {args.tokens} tokens a request in {s['rounds']} rounds, reward {s['reward'].item():.3f}, loss {s['loss'].item():.4f}")


if __name__ == "__main__":
    main()
