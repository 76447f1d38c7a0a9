"""A sentence classifier on the library's operators, the shape of the paper's 1-D text model ("CNN-non-static": the word
vectors are trained with the network): words -> vectors, channels first -> pruned 1-D convolutions spanning 2 and 3 words with bias
and ReLU -> the largest value of each filter over the sentence -> a fully connected layer in 8-bit integers.

    python -m paper_2011_06295_amd.text_model        # classifies synthetic sentences, then trains their word vectors
"""
from __future__ import annotations

import numpy as np
import torch
import torch.nn.functional as F

from . import binding as B
from . import text
from . import workloads as wl


class TextModel:
    """Filters are pruned and fixed, the classifier is quantised; the word vectors can be trained.  A gradient is that of the last
    forward: threads that train need a model each."""

    def __init__(self, table: torch.Tensor, filters, classifier: torch.Tensor, bias: torch.Tensor, padding: int = 0):
        """table: word vectors [vocab][dim], fp32.  filters: (weights [K][dim][1][S], mask, bias [K]) of each convolution, numpy
        arrays.  classifier [classes][sum of K], bias [classes].  padding: the token that sentences are filled up with."""
        self.words = text.Embedding(table, padding=padding)
        self.convs, self.transposed = [], []
        for weights, mask, conv_bias in filters:
            layer = B.SparseConv(weights, mask)
            layer.set_epilogue(conv_bias, relu=True)
            self.convs.append(layer)
            # the gradient of a convolution's input is the convolution with its filters turned round, channels and filters exchanged
            turned = [np.ascontiguousarray(a.transpose(1, 0, 2, 3)[..., ::-1]) for a in (weights, mask)]
            self.transposed.append(B.SparseConv(*turned))
        self.classifier = text.Int8Linear(classifier, bias)

    @classmethod
    def synthetic(cls, vocab: int = 20000, classes: int = 6, sparsity_bp: int = 8750, seed: int = 1, device: str = "cuda") -> "TextModel":
        """The sizes of the text workload (300 dimensions, 100 filters of each width), random weights."""
        gen = torch.Generator(device=device).manual_seed(seed)
        specs = [s for s in wl.cnn_1d().layers if s.sparsity_bp == sparsity_bp]
        filters = [(wl.make_weights(8, i, s), wl.make_mask(8, i, s), np.zeros(s.K, np.float32)) for i, s in enumerate(specs, 1)]
        table = torch.randn((vocab, specs[0].C), generator=gen, device=device)
        table[0] = 0.0
        features = sum(s.K for s in specs)
        return cls(table, filters, torch.randn((classes, features), generator=gen, device=device) / features ** 0.5, torch.zeros(classes, device=device))

    def forward(self, tokens: torch.Tensor) -> torch.Tensor:
        """Logits [sentences][classes] of tokens [sentences][words]; what the gradient needs is kept, the tokens as they are now."""
        x = self.words.forward(tokens, channels_first=True)
        self._tokens = tokens.clone()
        self._maps = [layer.forward(x) for layer in self.convs]
        best = [m.squeeze(2).max(2) for m in self._maps]
        self._places = [b.indices for b in best]
        return self.classifier.forward(torch.cat([b.values for b in best], 1))

    def vector_gradient(self, grad_logits: torch.Tensor) -> torch.Tensor:
        """Gradient [sentences][dim][1][words] of the vectors that the last forward looked up (rounding to 8 bits counts as the
        identity)."""
        grad_features = grad_logits @ self.classifier.dequantized()
        total, first = None, 0
        for layer, maps, places in zip(self.transposed, self._maps, self._places):
            count = maps.shape[1]
            g = grad_features[:, first:first + count]
            first += count
            largest = maps.squeeze(2).gather(2, places[..., None])[..., 0]
            grad_map = torch.zeros_like(maps).squeeze(2)
            grad_map.scatter_(2, places[..., None], (g * (largest > 0))[..., None])
            spread = layer.S - 1
            gx = layer.forward(F.pad(grad_map, (spread, spread))[:, :, None].contiguous())
            total = gx if total is None else total.add_(gx)
        return total

    def table_gradient(self, grad_logits: torch.Tensor) -> torch.Tensor:
        """Gradient [vocab][dim] of the word vectors."""
        return self.words.backward(self.vector_gradient(grad_logits), self._tokens, channels_first=True)

    def train_step(self, tokens: torch.Tensor, labels: torch.Tensor, rate: float) -> torch.Tensor:
        """One step of gradient descent on the word vectors; the loss before it.  Only rows that the sentences name are touched:
        -rate times their gradient is added to them in place."""
        logits = self.forward(tokens)
        p = torch.softmax(logits, 1)
        loss = -torch.log(p.gather(1, labels[:, None])).mean()
        p.scatter_add_(1, labels[:, None], torch.full_like(p, -1.0))
        grad = self.vector_gradient(p / len(tokens))
        table = self.words.table
        text.Embedding(table, scale=-rate, padding=self.words.padding).backward(grad, tokens, channels_first=True, out=table, accumulate=True)
        return loss

    def close(self):
        for layer in self.convs + self.transposed:
            layer.close()


def sentences(count: int = 128, words: int = 64, vocab: int = 20000, classes: int = 6, seed: int = 2, device: str = "cuda"):
    """(tokens [count][words] filled up with token 0, labels [count]) of synthetic sentences of 8 words and more."""
    gen = torch.Generator(device=device).manual_seed(seed)
    u = torch.rand((count, words), generator=gen, device=device, dtype=torch.float64)
    tokens = (float(vocab) ** u).long().clamp_(1, vocab - 1)
    length = torch.randint(8, words + 1, (count, 1), generator=gen, device=device)
    tokens[torch.arange(words, device=device)[None] >= length] = 0
    return tokens, torch.randint(0, classes, (count,), generator=gen, device=device)


def main() -> None:
    model = TextModel.synthetic()
    tokens, labels = sentences()
    print("classes of the first sentences:", model.forward(tokens)[:8].argmax(1).tolist())
    for step in range(20):
        loss = model.train_step(tokens, labels, rate=20.0)
        if step % 5 == 0:
            print(f"step {step}: loss {float(loss):.4f}")
    print(f"after training: loss {float(model.train_step(tokens, labels, rate=0.0)):.4f}, "
          f"right: {int((model.forward(tokens).argmax(1) == labels).sum())} of {len(labels)}")
    model.close()


if __name__ == "__main__":
    main()
