"""Features for the SVM: random cosine features, and a residual network that
is trained under the SVM's own squared hinge loss.

Both are made of the library's calls (``native.svm_linear`` and the others);
torch holds the memory.  Their outputs are dense float32 rows for
``native.svm_train`` and ``native.svm_train_ovr``.
"""
from __future__ import annotations

import math

import torch

from . import native as nv


class CosineFeatures:
    """Random Fourier features of the RBF kernel exp(-gamma |u - v|^2):
    phi(x) = cos(W x + b) with rows of W from N(0, 2 gamma I) and b from
    U[0, 2 pi); then (2/n) phi(u).phi(v) tends to the kernel as n grows, and
    an SVM with ``params()`` on phi to the RBF one on x."""

    def __init__(self, d: int, n: int, gamma: float, seed: int = 0,
                 dtype=torch.float32, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        W = torch.randn(n, d, generator=g) * math.sqrt(2.0 * gamma)
        b = torch.rand(n, generator=g) * (2.0 * math.pi)
        self.W, self.b = W.to(device, dtype), b.to(device, dtype)

    def __call__(self, X):
        return nv.svm_linear(X, self.W, self.b, act="cos")

    def params(self) -> dict:
        """Arguments of svm_train: K(u, v) = (2/n) u.v."""
        return dict(kernel=nv.SVM_KERNEL_POLY, degree=1, coef0=0.0,
                    gamma=2.0 / self.W.shape[0])


class FeatureNet:
    """x -> H0 = gelu(W0 x + b0), then blocks H + gelu(W norm(H) + b), and a
    linear head of class scores (one: two classes, label 1 against 0).

    ``step`` does one AdamW step on a batch under the squared hinge loss, one
    class against the rest; ``features`` are the last block's outputs, on
    which an SVM is trained in the head's place."""

    def __init__(self, d: int, width: int, blocks: int, classes: int,
                 dtype=torch.float32, bits: int = 32, seed: int = 0,
                 device="cuda"):
        g = torch.Generator().manual_seed(seed)

        def layer(n, k):
            return [(torch.randn(n, k, generator=g) / math.sqrt(k)).to(
                device, dtype), torch.zeros(n, dtype=dtype, device=device)]

        norm = lambda: [  # noqa: E731
            torch.ones(width, dtype=dtype, device=device),
            torch.zeros(width, dtype=dtype, device=device)]
        self.first = layer(width, d)
        self.blocks = [norm() + layer(width, width) for _ in range(blocks)]
        self.head = layer(classes, width)
        self.parameters = (self.first + [p for b in self.blocks for p in b]
                           + self.head)
        self.states = nv.svm_adamw_states(
            self.parameters, bits=bits, master=dtype != torch.float32)
        self.steps = 0

    def features(self, X):
        H = nv.svm_linear(X, *self.first, act="gelu")
        for w, c, W, b in self.blocks:
            N = nv.svm_layer_norm(H, w, c)
            H = nv.svm_linear(N, W, b, H, act="gelu", out=H)
        return H

    def scores(self, X):
        return nv.svm_linear(self.features(X), *self.head)

    def gradients(self, X, labels):
        """(loss, scores, gradients of the parameters in their order)."""
        H, Z0 = nv.svm_linear(X, *self.first, act="gelu", save=True)
        kept = []
        for w, c, W, b in self.blocks:
            N, mean, rstd = nv.svm_layer_norm(H, w, c, save=True)
            out, Z = nv.svm_linear(N, W, b, H, act="gelu", save=True)
            kept.append((H, N, mean, rstd, Z))
            H = out
        S = nv.svm_linear(H, *self.head)
        loss, dS = nv.svm_hinge_loss(S, labels)
        dH, dW, db = nv.svm_linear_backward(dS, H, self.head[0])
        grads = [dW, db]
        for (w, c, W, b), (H, N, mean, rstd, Z) in zip(self.blocks[::-1],
                                                       kept[::-1]):
            dN, dW, db = nv.svm_linear_backward(dH, N, W, Z, act="gelu")
            # what reaches H past the norm and the layer is dH itself
            dH, dw, dc = nv.svm_layer_norm_backward(dN, H, mean, rstd, w,
                                                    residual=dH)
            grads = [dw, dc, dW, db] + grads
        _, dW, db = nv.svm_linear_backward(dH, X, self.first[0], Z0,
                                           act="gelu",
                                           need=(False, True, True))
        return loss, S, [dW, db] + grads

    def step(self, X, labels, lr: float = 1e-3, weight_decay: float = 0.01):
        """One step on a batch -> its loss (a tensor on the device)."""
        loss, _, grads = self.gradients(X, labels)
        self.steps += 1
        nv.svm_adamw_step(self.parameters, grads, *self.states, lr=lr,
                          weight_decay=weight_decay, step=self.steps)
        return loss
