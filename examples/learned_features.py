#!/usr/bin/env python3
"""Features that the library makes, and SVMs trained on them.

1. Random cosine features of the benchmark's two Gaussians: an SVM on them
   against the RBF SVM that they stand for.
2. A residual feature network on the ten-class images, trained under the
   squared hinge loss in bfloat16 with 8-bit AdamW states, and a one-vs-rest
   SVM with a linear kernel on its features, against the same SVM on the
   images.

Synthetic data from paper_1706_05544_amd/workloads.py.  Needs the GPU.
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1706_05544_amd import native as nv  # noqa: E402
from paper_1706_05544_amd import workloads  # noqa: E402
from paper_1706_05544_amd.features import (CosineFeatures,  # noqa: E402
                                           FeatureNet)


def timed(what, f):
    torch.cuda.synchronize()
    t = time.perf_counter()
    out = f()
    torch.cuda.synchronize()
    print("  %-44s %8.1f ms" % (what, (time.perf_counter() - t) * 1e3))
    return out


def cosine(n, features):
    w = workloads.make("C3", n=n, n_test=n // 5)
    X, Xt = (torch.from_numpy(a).cuda() for a in (w.X, w.Xt))
    print("two Gaussians, %d x %d" % X.shape)
    rbf = timed("RBF SVM", lambda: nv.svm_train(X, w.y, C=w.C,
                                                gamma=w.gamma))
    phi = CosineFeatures(w.d, features, w.gamma)
    F, Ft = timed("%d cosine features" % features, lambda: (phi(X), phi(Xt)))
    lin = timed("SVM on them", lambda: nv.svm_train(F, w.y, C=w.C,
                                                    **phi.params()))
    acc = [float(np.mean(np.sign(D.cpu().numpy()) == w.yt))
           for D in (nv.svm_predict(rbf, Xt), nv.svm_predict(lin, Ft))]
    print("  accuracy: RBF %.4f, cosine features %.4f" % tuple(acc))
    return acc


def network(n, width, blocks, epochs, batch=512):
    w = workloads.make("C4", n=n, n_test=n // 5)
    X, Xt = (torch.from_numpy(a).cuda() for a in (w.X, w.Xt))
    labels = torch.from_numpy(w.y).cuda()
    print("ten classes of images, %d x %d" % X.shape)
    net = FeatureNet(w.d, width, blocks, w.n_classes, dtype=torch.bfloat16,
                     bits=8)
    Xb = X.bfloat16()
    order = torch.Generator(device="cuda").manual_seed(0)

    def epoch():
        losses = []
        for rows in torch.randperm(n, generator=order,
                                   device="cuda").split(batch):
            losses.append(net.step(Xb[rows], labels[rows], lr=1e-3))
        return torch.stack(losses).mean()

    for e in range(epochs):
        loss = timed("epoch %d" % (e + 1), epoch)
        print("    loss %.4f" % float(loss))
    F, Ft = timed("features", lambda: (net.features(Xb).float(),
                                       net.features(Xt.bfloat16()).float()))
    acc = []
    for what, A, At in (("images", X, Xt), ("features", F, Ft)):
        m = timed("one-vs-rest linear SVM on the " + what,
                  lambda: nv.svm_train_ovr(A, w.y, w.n_classes, C=0.01,
                                           kernel=nv.SVM_KERNEL_LINEAR))
        acc.append(float(np.mean(nv.svm_predict_labels(m, At).cpu().numpy()
                                 == w.yt)))
    print("  accuracy: images %.4f, features %.4f" % tuple(acc))
    return acc


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--n", type=int, default=20000)
    ap.add_argument("--features", type=int, default=2048)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--epochs", type=int, default=3)
    a = ap.parse_args()
    cosine(a.n, a.features)
    network(a.n, a.width, a.blocks, a.epochs)
