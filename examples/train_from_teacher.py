"""Training a joint's output layer from a teacher that decodes with phrase lists.

A teacher joint (a random layer over synthetic frame features) decodes a batch
of streams with boosting; its frames are scored (how likely was each emitted
token without boosting, how sure was the teacher, what else was likely), and a
student layer learns from the teacher's alternatives with their tail, plus the
log-likelihood of the decoded tokens, weighted by the teacher's confidence.

    python examples/train_from_teacher.py [--steps 30]
"""

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np  # noqa: E402
import torch  # noqa: E402

from paper_2608_21343_amd.decoder import BoostDecoder  # noqa: E402
from paper_2608_21343_amd.optim import AdamW  # noqa: E402
from paper_2608_21343_amd.rowops import distill_loss, token_scores  # noqa: E402


def main(steps: int = 30, B: int = 32, T: int = 64, V: int = 1024, width: int = 256,
         n_alt: int = 16, temperature: float = 1.5, seed: int = 0, quiet: bool = False):
    """Mean loss of the first and the last step."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    frames = normal(T, B, width)
    teacher = normal(V + 1, width) * (3.0 / width ** 0.5)

    # decode with a phrase list per stream
    rng = np.random.default_rng(seed)
    lists = [[rng.integers(0, V, size=3).astype(np.int32) for _ in range(50)] for _ in range(B)]
    classes = np.arange(V + 1, dtype=np.int32)
    classes[V] = -1
    decoder = BoostDecoder(lists, classes)
    logits = frames @ teacher.T
    mids, states, _ = decoder.start(range(B))
    tokens, _, _ = decoder.greedy(logits, mids, states)

    # what the teacher thought of every frame
    seen = token_scores(logits, tokens, n_alt=n_alt, temperature=temperature)
    boosted = tokens != seen.alt[..., 0]
    sure = torch.exp(-seen.entropy)
    weight = sure / sure.sum()
    if not quiet:
        print(f"{B * T} frames, {int(boosted.sum())} decided by boosting, "
              f"mean entropy {float(seen.entropy.mean()):.2f}")

    # learn from its alternatives and from what was decoded
    student = torch.zeros((V + 1, width), device="cuda", requires_grad=True)
    optimizer = AdamW([student], lr=0.02, weight_decay=0.0)
    losses = []
    for step in range(steps):
        z = (frames.reshape(-1, width) @ student.T).view(T, B, V + 1)
        soft = distill_loss(z, seen.alt, seen.alt_logprob, temperature=temperature, tail=True,
                            weight=weight)
        hard = token_scores(z, tokens).logprob * weight
        loss = soft.sum() - 0.1 * hard.sum()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(float(loss.detach()))
        if not quiet and step % 10 == 0:
            print(f"step {step}: loss {losses[-1]:.4f}")
    if not quiet:
        agree = (z.argmax(-1) == logits.argmax(-1)).float().mean()
        print(f"last loss {losses[-1]:.4f}, best token agrees in {100 * float(agree):.0f}% of frames")
    return losses[0], losses[-1]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__)
    ap.add_argument("--steps", type=int, default=30)
    main(ap.parse_args().steps)
