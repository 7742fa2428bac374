"""Features for the SVM: random cosine features, and a residual network that
is trained under the SVM's own squared hinge loss and served in 4-bit weights.

Both are made of the library's calls (``native.svm_linear`` and the others);
torch holds the memory.  Their outputs are dense float32 rows for
``native.svm_train`` and ``native.svm_train_ovr``.
"""
from __future__ import annotations

import math
from typing import Optional

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


def patches(X, side: int, size: int):
    """Rows of side x side images cut into size x size patches: (images,
    patches, size^2)."""
    n, k = X.shape[0], side // size
    X = X.reshape(n, k, size, k, size).transpose(2, 3)
    return X.reshape(n, k * k, size * size)


class _Network:
    """What a network's layers make of X, in training and served."""

    def features(self, X):
        H = self._layer(X, self.first, act="gelu")
        for w, c, *layer in self.blocks:
            if self.groups:
                N = nv.svm_group_norm(H, self.groups, w, c, act="gelu")
                H = self._layer(N, layer, H, out=H)
            else:
                N = nv.svm_layer_norm(H, w, c)
                H = self._layer(N, layer, H, act="gelu", out=H)
        return H.flatten(1) if self.groups else H

    def scores(self, X):
        return self._layer(self.features(X), self.head)


class FeatureNet(_Network):
    """x -> H0 = gelu(W0 x + b0), then blocks H + gelu(W norm(H) + b), and a
    linear head of class scores (one: two classes, label 1 against 0).

    With ``groups`` a sample is ``positions`` rows of d values (an image's
    patches, say) that share the layers, and a block is
    H + W gelu(group_norm(H)) + b with the statistics over all positions; the
    features are all positions' outputs side by side.

    ``step`` does one AdamW step on a batch under the squared hinge loss, one
    class against the rest; ``features`` are the last block's outputs, on
    which an SVM is trained in the head's place; ``packed`` is the network in
    4-bit weights, to be served."""

    def __init__(self, d: int, width: int, blocks: int, classes: int,
                 dtype=torch.float32, bits: int = 32, seed: int = 0,
                 device="cuda", groups: int = 0, positions: int = 1):
        g = torch.Generator().manual_seed(seed)

        def layer(n, k):
            return [(torch.randn(n, k, generator=g) / math.sqrt(k)).to(
                device, dtype), torch.zeros(n, dtype=dtype, device=device)]

        norm = lambda: [  # noqa: E731
            torch.ones(width, dtype=dtype, device=device),
            torch.zeros(width, dtype=dtype, device=device)]
        self.groups = groups
        self.first = layer(width, d)
        self.blocks = [norm() + layer(width, width) for _ in range(blocks)]
        self.head = layer(classes, width * (positions if groups else 1))
        self.parameters = (self.first + [p for b in self.blocks for p in b]
                           + self.head)
        self.states = nv.svm_adamw_states(
            self.parameters, bits=bits, master=dtype != torch.float32)
        self.steps = 0       # asked for
        # of them, those whose gradients were not finite (on the device)
        self.left_out = torch.zeros((), dtype=torch.int64, device=device)
        self.norm = None  # of the last clipped step's gradients

    @staticmethod
    def _layer(X, layer, residual=None, act="none", out=None):
        return nv.svm_linear(X, *layer, residual, act=act, out=out)

    def packed(self, group: int = 64) -> "PackedNet":
        return PackedNet(self, group)

    def gradients(self, X, labels):
        """(loss, scores, gradients of the parameters in their order)."""
        H, Z0 = nv.svm_linear(X, *self.first, act="gelu", save=True)
        kept = []
        for w, c, W, b in self.blocks:
            if self.groups:
                N, mean, rstd = nv.svm_group_norm(H, self.groups, w, c,
                                                  act="gelu", save=True)
                out, Z = nv.svm_linear(N, W, b, H), None
            else:
                N, mean, rstd = nv.svm_layer_norm(H, w, c, save=True)
                out, Z = nv.svm_linear(N, W, b, H, act="gelu", save=True)
            kept.append((H, N, mean, rstd, Z))
            H = out
        F = H.flatten(1) if self.groups else H
        S = nv.svm_linear(F, *self.head)
        loss, dS = nv.svm_hinge_loss(S, labels)
        dH, dW, db = nv.svm_linear_backward(dS, F, self.head[0])
        dH = dH.view(H.shape)
        grads = [dW, db]
        for (w, c, W, b), (H, N, mean, rstd, Z) in zip(self.blocks[::-1],
                                                       kept[::-1]):
            dN, dW, db = nv.svm_linear_backward(
                dH, N, W, Z, act="none" if self.groups else "gelu")
            # what reaches H past the norm and the layer is dH itself
            if self.groups:
                dH, dw, dc = nv.svm_group_norm_backward(
                    dN, H, self.groups, mean, rstd, w, c, act="gelu",
                    residual=dH)
            else:
                dH, dw, dc = nv.svm_layer_norm_backward(dN, H, mean, rstd, w,
                                                        residual=dH)
            grads = [dw, dc, dW, db] + grads
        _, dW, db = nv.svm_linear_backward(dH, X, self.first[0], Z0,
                                           act="gelu",
                                           need=(False, True, True))
        return loss, S, [dW, db] + grads

    def step(self, X, labels, lr: float = 1e-3, weight_decay: float = 0.01,
             clip: Optional[float] = None):
        """One step on a batch -> its loss (a tensor on the device).  With
        ``clip`` the gradients' norm is brought down to it, and kept in
        ``norm`` (on the device); a step whose gradients are not finite
        changes nothing but ``left_out``, and the steps after it are as if it
        had never been."""
        loss, _, grads = self.gradients(X, labels)
        self.steps += 1
        factor = None
        if clip is not None:
            self.norm, factor = nv.svm_grad_norm(grads, clip)
        nv.svm_adamw_step(self.parameters, grads, *self.states, lr=lr,
                          weight_decay=weight_decay, step=self.steps,
                          factor=factor, left_out=self.left_out)
        return loss


class PackedNet(_Network):
    """A FeatureNet's layers in 4 bits, with copies of its norms and biases:
    what ``features`` and ``scores`` of a request need, and nothing that
    training the network on would change.  A weight takes 4 bits and its share
    of a scale, in whole tiles of 16 outputs by 128 inputs: in groups of 64, a
    seventh of the float32 weights' memory and somewhat over a quarter of the
    16-bit ones'."""

    def __init__(self, net: FeatureNet, group: int = 64):
        pack = lambda layer: [  # noqa: E731
            nv.svm_pack_weights(layer[0], group), layer[1].clone()]
        self.groups = net.groups
        self.first = pack(net.first)
        self.blocks = [[p.clone() for p in b[:2]] + pack(b[2:])
                       for b in net.blocks]
        self.head = pack(net.head)

    @staticmethod
    def _layer(X, layer, residual=None, act="none", out=None):
        return nv.svm_linear_packed(X, *layer, residual, act=act, out=out)
