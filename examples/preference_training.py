"""From a teacher and pairs of answers to a policy, with one solver and four losses.

  1. A student head learns a teacher's distribution from its top logits (distill_loss).
  2. A reward model, Bradley-Terry over the answers' mean features, is fitted to the pairs in a box by the L-BFGS-B solver
     (OBJ_LOGISTIC_L2 on differences of features).
  3. The head learns the pairs themselves (token_logprob -> preference_loss -> token_logprob_grad), against the distilled head.
  4. The head is trained on its own samples, scored by the reward model, with the clipped policy loss (policy_loss).

The body of the model stands still: random features of every position; what is trained is the head that turns them into
logits, by torch's optimizer, which gets the losses' gradients through `logits.backward(r.grad)`.

    python examples/preference_training.py [--vocab 4096] [--width 64] [--pairs 64]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2203_16340_amd as L  # noqa: E402


def make_task(vocab, width, pairs, tokens, gen, device):
    """Features of every token of 2 * pairs answers, a teacher's head, a token for every position, and a hidden taste that
    says which answer of a pair was chosen."""
    def randn(*shape):
        return torch.randn(*shape, device=device, generator=gen)

    lengths = torch.randint(tokens // 2, tokens + 1, (2 * pairs,), device=device, generator=gen)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=device), torch.cumsum(lengths, 0)])
    total = int(offsets[-1])
    answer = torch.repeat_interleave(torch.arange(2 * pairs, device=device), lengths)
    # (an answer has a direction of its own, so that answers differ as a whole)
    features = randn(total, width) + randn(2 * pairs, width)[answer]
    teacher = randn(vocab, width) * 0.4
    labels = torch.distributions.Categorical(logits=features @ teacher.t()).sample()
    mean = torch.zeros(2 * pairs, width, device=device).index_add_(0, answer, features) / lengths[:, None]
    taste = randn(width)
    score = mean @ taste
    # put the answers in order: chosen ones first
    swap = score[:pairs] < score[pairs:]
    first = torch.where(swap, torch.arange(pairs, device=device) + pairs, torch.arange(pairs, device=device))
    order = torch.cat([first, (first + pairs) % (2 * pairs)])
    at = torch.cat([torch.arange(int(offsets[k]), int(offsets[k + 1]), device=device) for k in order.tolist()])
    offsets = torch.cat([offsets[:1], torch.cumsum(lengths[order], 0)])
    return dict(features=features[at], labels=labels[at], offsets=offsets, mean=mean[order], teacher=teacher)


def distill(head, task, top, steps, lr):
    full = task["features"] @ task["teacher"].t()
    a, index = torch.topk(full, top, dim=1)
    lse = torch.logsumexp(full, 1)                      # what the top logits leave out is one more outcome
    mean = torch.full((len(a),), 1.0 / len(a), device=a.device)
    opt, losses = torch.optim.Adam(head.parameters(), lr=lr), []
    for _ in range(steps):
        logits = head(task["features"])
        r = L.distill_loss(logits.detach(), index, a, teacher_lse=lse, weight=mean)
        opt.zero_grad()
        logits.backward(r.grad)
        opt.step()
        losses.append(r.loss)
    return torch.stack(losses).tolist()


def fit_reward(task, bound=8.0, mu=1e-3):
    """Bradley-Terry: minimise mean softplus(-(w . (chosen - rejected))) + mu/2 |w|^2 over -bound <= w <= bound."""
    pairs = len(task["mean"]) // 2
    A = (task["mean"][:pairs] - task["mean"][pairs:]).double().contiguous()
    n, dev = A.shape[1], A.device
    box = torch.full((n,), bound, dtype=torch.float64, device=dev)
    with L.Solver(L.OBJ_LOGISTIC_L2, A, torch.ones(pairs, dtype=torch.float64, device=dev), -box, box, 10, mu=mu,
                  options=L.default_options(tol=1e-7)) as s:
        s.set_x(torch.zeros(n, dtype=torch.float64, device=dev))
        info = s.solve()
        return s.x().float(), info


def prefer(head, task, steps, lr, beta):
    with torch.no_grad():
        ref = L.token_logprob(head(task["features"]), task["labels"]).logp
    pairs = len(task["offsets"]) // 2
    mean = torch.full((pairs,), 1.0 / pairs, device=ref.device)
    opt, losses = torch.optim.Adam(head.parameters(), lr=lr), []
    for _ in range(steps):
        logits = head(task["features"])
        z = logits.detach()
        t = L.token_logprob(z, task["labels"])
        r = L.preference_loss(t.logp, ref, task["offsets"], weight=mean, beta=beta, length_normalised=True)
        opt.zero_grad()
        logits.backward(L.token_logprob_grad(z, task["labels"], t, r.grad))
        opt.step()
        losses.append(r.loss)
    right = (r.rewards[:pairs] > r.rewards[pairs:]).float().mean().item()
    return torch.stack(losses).tolist(), right


def improve(head, task, reward, rounds, steps, lr, gen):
    """Samples a token for every position; a token's reward is what the reward model gives the teacher's direction of it."""
    x = task["features"]
    value = task["teacher"] @ reward                    # the reward of each token of the vocabulary
    value = (value - value.mean()) / value.std()
    with torch.no_grad():
        ref_head = head(x).detach()
    mean = torch.full((len(x),), 1.0 / len(x), device=x.device)
    opt, rewards = torch.optim.Adam(head.parameters(), lr=lr), []
    for _ in range(rounds):
        with torch.no_grad():
            z = head(x)
            noise = -torch.log(-torch.log(torch.rand(z.shape, device=z.device, generator=gen).clamp(1e-9, 1 - 1e-7)))
            y = torch.argmax(z + noise, 1)
            old, ref = L.token_logprob(z, y).logp, L.token_logprob(ref_head, y).logp
        got = value[y]
        rewards.append(got.mean().item())
        adv = ((got - got.mean()) / got.std()).contiguous()
        for _ in range(steps):
            logits = head(x)
            r = L.policy_loss(logits.detach(), y, old, adv, ref_logp=ref, weight=mean, kl_coef=0.02, entropy_coef=1e-3)
            opt.zero_grad()
            logits.backward(r.grad)
            opt.step()
    return rewards


def run(vocab=4096, width=64, pairs=64, tokens=24, seed=0, device="cuda:0"):
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    torch.manual_seed(seed)
    task = make_task(vocab, width, pairs, tokens, gen, device)
    head = torch.nn.Linear(width, vocab, bias=False, device=device)
    out = {"distill": distill(head, task, 64, 60, 0.02)}
    reward, info = fit_reward(task)
    pairs_right = (task["mean"][:pairs] @ reward > task["mean"][pairs:] @ reward).float().mean().item()
    out.update(reward_status=info.status, reward_iterations=info.iters, reward_right=pairs_right)
    out["preference"], out["preference_right"] = prefer(head, task, 30, 0.002, 1.0)
    out["policy"] = improve(head, task, reward, 8, 4, 0.01, gen)
    return out


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("vocab", 4096), ("width", 64), ("pairs", 64), ("tokens", 24), ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=default)
    r = run(**vars(ap.parse_args()))
    print(f"distillation: {r['distill'][0]:.3f} -> {r['distill'][-1]:.3f}")
    print(f"reward model: {r['reward_iterations']} iterations, {100 * r['reward_right']:.0f} % of the pairs in order")
    print(f"preference loss: {r['preference'][0]:.3f} -> {r['preference'][-1]:.3f}, {100 * r['preference_right']:.0f} % of the pairs in order")
    print("reward of samples: " + " ".join(f"{v:.3f}" for v in r["policy"]))


if __name__ == "__main__":
    main()
