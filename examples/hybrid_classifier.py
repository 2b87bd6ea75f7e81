"""A hybrid classifier: classical layers around a variational circuit, trained end to end.

    features -> layer norm -> linear, tanh -> angles -> circuit -> <Z> -> linear -> logits
             -> log probabilities of the labels

Every step of the forward and the backward runs in the library's kernels; torch holds the
parameters, chains the gradients and runs the optimizer.  After the training the outcome
probabilities of a few states are scored the same way: log probabilities of measured shots,
entropy, and the likeliest outcomes.

    python examples/hybrid_classifier.py --qubits 8 --steps 200
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_11985_amd import layers  # noqa: E402
from paper_2607_11985_amd import workloads as W  # noqa: E402
from paper_2607_11985_amd.api import Circuit, VQCFunction  # noqa: E402


def synthetic(batch, features, classes, generator, device):
    """Labelled points around one centre per class."""
    centres = torch.randn((classes, features), generator=generator)
    labels = torch.randint(0, classes, (batch,), generator=generator)
    points = centres[labels] + 0.7 * torch.randn((batch, features), generator=generator)
    return points.to(device), labels.to(device)


class Hybrid:
    """Parameters and forward pass; the circuit is a hardware-efficient ansatz behind one angle
    per qubit, its parameters shared by the batch."""

    def __init__(self, features, classes, qubits, depth, generator, device):
        ops, n_params, n_inputs = W.hea_circuit(qubits, depth)
        self.circuit = Circuit(ops, qubits, n_params, n_inputs, device=device.index or 0,
                               shared_params=True)

        def param(*shape, scale=1.0, offset=0.0):
            t = torch.randn(shape, generator=generator) * scale + offset
            return t.to(device).requires_grad_(True)

        self.norm_w = param(features, scale=0.0, offset=1.0)
        self.norm_b = param(features, scale=0.0)
        self.enc_w = param(n_inputs, features, scale=features ** -0.5)
        self.enc_b = param(n_inputs, scale=0.0)
        self.theta = param(n_params, scale=0.3)
        self.out_w = param(classes, qubits, scale=1.0)
        self.out_b = param(classes, scale=0.0)

    def parameters(self):
        return [self.norm_w, self.norm_b, self.enc_w, self.enc_b, self.theta, self.out_w,
                self.out_b]

    def angles(self, x):
        h = layers.layer_norm(x, self.norm_w, self.norm_b)
        return math.pi * layers.linear(h, self.enc_w, self.enc_b, "tanh")

    def logits(self, x):
        expectations = VQCFunction.apply(self.circuit, self.theta, self.angles(x))
        return layers.linear(expectations, self.out_w, self.out_b)


def train(steps=100, batch=256, features=64, classes=4, qubits=8, depth=2, seed=0, report=None):
    """Trains on one synthetic set; returns the model, its data and the losses."""
    device = torch.device("cuda", 0)
    generator = torch.Generator().manual_seed(seed)
    x, labels = synthetic(batch, features, classes, generator, device)
    model = Hybrid(features, classes, qubits, depth, generator, device)
    optimizer = torch.optim.Adam(model.parameters(), lr=0.05)
    losses = []
    for step in range(steps):
        optimizer.zero_grad()
        scores = layers.log_probs(model.logits(x), labels)
        loss = -scores.logp.mean()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
        if report and step % report == 0:
            print(f"step {step}: loss {float(losses[-1]):.4f}, entropy "
                  f"{float(scores.entropy.detach().mean()):.4f}", flush=True)
    return model, x, labels, torch.stack(losses).cpu()


@torch.no_grad()
def score_outcomes(model, x, shots=16, top=3, seed=0):
    """Measured shots of the encoded states: their log probabilities, the entropy of the outcome
    distribution and its likeliest outcomes."""
    angles = model.angles(x)
    _, probs = model.circuit.forward_ex(model.theta.detach(), angles, expvals=False, probs=True)
    generator = torch.Generator(device=probs.device).manual_seed(seed)
    measured = torch.multinomial(probs, shots, replacement=True, generator=generator)
    return layers.log_probs(probs, measured, top=top, kind="weights")


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--qubits", type=int, default=8)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=256)
    a = ap.parse_args()
    model, x, labels, _ = train(steps=a.steps, batch=a.batch, qubits=a.qubits, report=20)
    with torch.no_grad():
        scores = layers.log_probs(model.logits(x), labels, top=1)
    right = (scores.top_index.squeeze(-1) == labels).float().mean()
    print(f"trained: loss {float(-scores.logp.mean()):.4f}, accuracy {float(right):.3f}")
    s = score_outcomes(model, x[:2])
    for b in range(2):
        print(f"state {b}: entropy {float(s.entropy[b]):.3f}, shots' mean log probability "
              f"{float(s.logp[b].mean()):.3f}, likeliest outcomes {s.top_index[b].tolist()}")


if __name__ == "__main__":
    main()
