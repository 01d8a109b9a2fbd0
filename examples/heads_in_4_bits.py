"""Workers that train output layers in 4-bit products and gossip them.

Every worker holds an output layer W [V][K] and hidden states x [T][K] of its
own.  The tokens to predict are sampled from a teacher layer's predictions.
An inner step quantises W, forms the logits x W^T, and takes the gradients of
the mean cross-entropy from 4-bit products again; an outer step mixes the
workers' layers over a ring and applies the Nesterov update.  After each round
the workers' predictions are compared with the averaged layer's (the
Jensen-Shannon distance), and the averaged layer samples tokens.

    python examples/heads_in_4_bits.py
    python examples/heads_in_4_bits.py --workers 8 --vocab 32000 --width 1024 --tokens 512 --rounds 4
"""

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2606_22768_amd as fgd  # noqa: E402
from synth import configs  # noqa: E402


def cross_entropy(logits, targets):
    """Mean cross-entropy of logits [M][T][V] and its gradient in bf16."""
    z = logits.float()
    logp = z - torch.logsumexp(z, dim=-1, keepdim=True)
    picked = targets.long().unsqueeze(-1)
    loss = -logp.gather(-1, picked).mean()
    dy = logp.exp_()
    dy.scatter_add_(-1, picked, -torch.ones_like(picked, dtype=torch.float32))
    return loss, (dy / logits.shape[1]).bfloat16()


def train(workers=4, vocab=2000, width=256, tokens=128, rounds=5, inner_steps=8, lr=8.0, temperature=0.7, top_p=0.95,
          seed=0):
    """One dict per round: the loss before it, the workers' distance, and what
    the averaged layer samples."""
    M, V, K, T = workers, vocab, width, tokens
    dev = torch.device("cuda", 0)
    rng = torch.Generator(device=dev).manual_seed(seed)

    engine = fgd.Engine(M, V * K, V * K, "f32", outer_lr=0.7, momentum=0.9, device=0)
    state = engine.alloc_state()
    before, local = state["theta_prev"], state["theta_local"]
    before.zero_()
    state["momentum"].zero_()
    heads = local.view(M, V, K)
    engine.set_topology("mix1", "global")
    engine.set_topology_dict("mix2", configs.topology(("ring", "metropolis", 0.1), M, 1, seed=seed, step=0))

    teacher = fgd.mx4_quantize(torch.randn(V, K, device=dev, generator=rng) * (4.0 / K ** 0.5))
    x = torch.randn(M, T, K, device=dev, generator=rng).bfloat16()
    held_out = torch.randn(T, K, device=dev, generator=rng).bfloat16()
    targets, _ = fgd.sample(fgd.mx4_linear(x.view(M * T, K), teacher), torch.rand(M * T, device=dev, generator=rng))
    targets = targets.view(M, T)
    x_t = fgd.mx4_quantize(x.mT)  # of the weights' gradient: the same in every step

    ldk = (V + 7) // 8 * 8  # the distance reads rows of whole 16 bytes
    own = torch.zeros(M, T, ldk, dtype=torch.bfloat16, device=dev)
    average = torch.zeros(T, ldk, dtype=torch.bfloat16, device=dev)

    report = []
    for _ in range(rounds):
        local.copy_(before)
        first = None
        for _ in range(inner_steps):
            heads4, heads_t = fgd.mx4_quantize_both(heads)
            logits = fgd.mx4_linear(x, heads4)
            loss, dy = cross_entropy(logits, targets)
            first = loss if first is None else first
            _, dw = fgd.mx4_linear_grads(dy, x_t, heads_t)
            heads.sub_(dw, alpha=lr)
        # The workers' own predictions of the same states, and their average's.
        fgd.mx4_linear(held_out.expand(M, T, K), fgd.mx4_quantize(heads), out=own[..., :V])
        fgd.mx4_linear(held_out, fgd.mx4_quantize(heads.mean(0)), out=average[..., :V])
        distance, _ = fgd.js_distance(average, own, top_k=min(100, V), vocab=V)
        drawn, probs = fgd.sample(average, torch.rand(T, device=dev, generator=rng), temperature, top_p=top_p,
                                  vocab=V)
        engine.outer_step(before, local, state["momentum"])
        report.append(dict(loss=first, distance=distance.mean(), tokens=drawn, probs=probs))
    engine.close()
    return [dict(loss=float(r["loss"]), distance=float(r["distance"]), tokens=r["tokens"].cpu(),
                 probs=r["probs"].cpu()) for r in report]


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("workers", 4), ("vocab", 2000), ("width", 256), ("tokens", 128), ("rounds", 5),
                        ("inner-steps", 8), ("seed", 0)):
        p.add_argument(f"--{name}", type=int, default=value)
    for name, value in (("lr", 8.0), ("temperature", 0.7), ("top-p", 0.95)):
        p.add_argument(f"--{name}", type=float, default=value)
    for i, r in enumerate(train(**{k.replace("-", "_"): v for k, v in vars(p.parse_args()).items()})):
        print(f"round {i}: loss {r['loss']:.4f}  JS distance {r['distance']:.3e}  tokens "
              f"{r['tokens'][:6].tolist()}  with probability {r['probs'][:6].mean():.3f}", flush=True)


if __name__ == "__main__":
    main()
