"""A map of dense documents: a projection of language-model states is trained towards
the units of a codebook, then served in 8 bits.

    python examples/dense_map.py [--steps 40] [--docs 2048] [--states 1024] [--side 32] [--features 512]
                                 [--given] [--orthogonal] [--blocks]

The layer is norm(states + residual) -> product with bias and gelu -> dropout; its
output is a document in the map's feature space, whose distances to the units are
one product with the codebook: |z|^2 + |w_j|^2 - 2 z.w_j (scaled by -2, the codebook's
norms as bias).  The loss is the mean distance to the nearest unit; its gradient goes
back through dropout, the product and the norm.  Serving normalises straight into 8
bits and multiplies with 8-bit weights laid out by unit.

With --given every document has its unit (here the one that the untrained layer finds) and the loss is
the cross entropy of minus its scaled distances to all units; with --orthogonal the weights
move by their gradient orthogonalised, all directions alike; with --blocks serving uses a factor for each
block of 128 instead of one for each row."""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_05138_amd as som  # noqa: E402


class Layer:
    """The projection's weights, in half precision with fp32 copies that are trained."""

    def __init__(self, states, features, generator, dropout=0.1, dtype=torch.float16, device="cuda"):
        self.dtype, self.dropout, self.seed = dtype, dropout, 1234
        self.gain = torch.ones(states, device=device)
        self.W = torch.randn((states, features), generator=generator, device=device) * states ** -0.5
        self.bias = torch.zeros(features, device=device)

    def half(self):
        return self.gain.to(self.dtype), self.W.to(self.dtype)

    def forward(self, x, residual, step=None):
        """The documents, and what the gradient needs; step None: without dropout."""
        gain, W = self.half()
        y, h, _ = som.som_rms_norm(x, gain, residual=residual)
        pre = torch.empty((x.shape[0], W.shape[1]), dtype=self.dtype, device=x.device)
        z = som.som_product(y, W, bias=self.bias, act="gelu", pre=pre)
        if step is not None:
            z = som.som_dropout(z, self.dropout, self.seed, step)
        return z, (h, y, pre, gain, W, step)

    def backward(self, dz, kept, scale, rate, orthogonal=False):
        """One step down the gradient dz / scale (scaled so that half precision holds it); orthogonal: the
        weights by a matrix whose singular values are all about rate / 10."""
        h, y, pre, gain, W, step = kept
        dz = som.som_dropout(dz, self.dropout, self.seed, step)
        dy, dW, dbias = som.som_product_backward(dz, y, W, act="gelu", pre=pre)
        _, dgain = som.som_rms_norm_backward(dy, h, gain)
        self.W -= 0.1 * rate * som.som_orthogonalise(dW).float() if orthogonal else rate / scale * dW.float()
        self.bias -= rate / scale * dbias
        self.gain -= rate / scale * dgain

    def quantised(self):
        """8-bit weights laid out by unit, and a factor for each."""
        W = self.W.t().contiguous()
        scale = W.abs().amax(1) / 448.0
        return (W / scale[:, None]).to(torch.float8_e4m3fn).t(), scale


    def quantised_blocks(self):
        """8-bit weights laid out by unit, and a factor for each block of 128 x 128."""
        q, scale = som.som_quantise(self.W, 128, transpose=True)
        return q.t(), scale


def given_loss(z, codebook, N, norms, units, t, scale):
    """(mean cross entropy of the documents' units by -t |z - w_j|^2, its gradient by z times scale)."""
    docs = z.shape[0]
    W, bias = codebook[:, :N], -t * norms          # |z|^2 is the same for all units
    loss, lse = som.som_cross_entropy(z, W, units, bias=bias, alpha=2.0 * t)
    dloss = torch.full((docs,), scale / docs, device=z.device)
    dz, _, _ = som.som_cross_entropy_backward(dloss, z, W, units, lse, bias=bias, alpha=2.0 * t, need_dW=False,
                                              need_dbias=False)
    return loss.mean(), dz


def nearest(z, codebook, N, norms):
    """(unit, squared distance) of every document."""
    scores = som.som_product(z, codebook[:, :N], bias=norms, alpha=-2.0, dtype=torch.float32)
    least, unit = scores.min(1)
    return unit, least + (z.float() ** 2).sum(1)


def main(steps=40, docs=2048, states=1024, side=32, features=512, rate=0.3, seed=0, say=print, given=False,
         orthogonal=False, blocks=False):
    """Returns the losses and the share of documents whose unit is the same in 8 bits."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    N = side * side
    codebook = torch.zeros((features, som.som_codebook_ldw(N)), dtype=torch.float16, device="cuda")
    codebook[:, :N] = torch.rand((features, N), generator=g, device="cuda").half()
    norms = som.som_codebook_norms(codebook, N=N)
    x = torch.randn((docs, states), generator=g, device="cuda").half()
    residual = torch.randn((docs, states), generator=g, device="cuda").half()
    layer = Layer(states, features, g)
    losses = []
    units = nearest(layer.forward(x, residual)[0], codebook, N, norms)[0].int() if given else None
    for step in range(steps):
        z, kept = layer.forward(x, residual, step)
        scale = float(docs)
        if given:
            loss, dz = given_loss(z, codebook, N, norms, units, 16.0 / features, scale)
            losses.append(float(loss))
        else:
            unit, distance = nearest(z, codebook, N, norms)
            losses.append(float(distance.mean()))
            # d(mean distance)/dz = 2 (z - w) / docs; the sum's gradient over features keeps its size
            dz = (2.0 * (z.float() - codebook.t()[unit].float()) * (scale / docs)).half()
        layer.backward(dz, kept, scale, rate, orthogonal)
        if step % 10 == 0 or step == steps - 1:
            say(f"step {step}: mean {'cross entropy' if given else 'squared distance'} {losses[-1]:.3f}")
    z, _ = layer.forward(x, residual)
    unit, distance = nearest(z, codebook, N, norms)
    if blocks:
        W8, scale8 = layer.quantised_blocks()
        y8, row_scale = som.som_quantise(som.som_rms_norm(x, layer.gain.half(), residual=residual)[0])
        z8 = som.som_product_blocks(y8, row_scale, W8, scale8, bias=layer.bias, act="gelu", dtype=torch.float16)
    else:
        W8, scale8 = layer.quantised()
        y8, _, row_scale = som.som_rms_norm(x, layer.gain.half(), residual=residual, q8=True)
        z8 = som.som_product(y8, W8, bias=layer.bias, act="gelu", x_scale=row_scale, w_scale=scale8, dtype=torch.float16)
    unit8, distance8 = nearest(z8, codebook, N, norms)
    same = float((unit8 == unit).float().mean())
    say(f"without dropout: {float(distance.mean()):.3f}; served in 8 bits: {float(distance8.mean()):.3f}, "
        f"{100 * same:.1f}% of the documents at the same unit")
    one, _ = nearest(layer.forward(x[:1], residual[:1])[0], codebook, N, norms)      # a single document
    say(f"document 0 alone: unit {int(one)} (in the batch {int(unit[0])})")
    return losses, same


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("steps", 40), ("docs", 2048), ("states", 1024), ("side", 32), ("features", 512)):
        ap.add_argument("--" + name, type=int, default=value)
    for name in ("given", "orthogonal", "blocks"):
        ap.add_argument("--" + name, action="store_true")
    a = ap.parse_args()
    main(a.steps, a.docs, a.states, a.side, a.features, given=a.given, orthogonal=a.orthogonal, blocks=a.blocks)
