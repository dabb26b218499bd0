"""How far a greedy text is from what the toy model of examples/drafted_trees.py says, token by token, in 64 bits; and how far the roundings of the attention can bring it.

A kernel's O differs from the exact one by the rounding of its bf16 result, at most 2^-8 of an element, and of the weights, at most 2^-8 of each: both taken as independent and evenly distributed, so
with a standard deviation of 1 / sqrt(3) of that.  What they do to the difference of two tokens' scores, whose columns of the output matrix differ by d, is the root of the sum of
(2^-8 O_i d_i)^2 / 3 over the columns and of (2^-8 w_hj v_hj . d_h)^2 / 3 over heads and keys.  SIGMAS of that are allowed (a chance of 2e-9 a token), and beside it what 32-bit sums may be off:
a product of up to 128 terms that add up to some 26 in the exponent, 128 * 2^-24 * 26 = 2e-4 < 2^-12 of a weight, and 1024 terms of the scores, 1024 * 2^-24 = 2^-14 of their magnitude."""
import math

import torch

SIGMAS = 6.0


def through_the_cache(x, codes, scale=0.0125):
    """rows as the cache gives them back, float64"""
    if not codes:
        return x.double()
    return (x.float() / torch.tensor(scale)).clamp(-448, 448).to(torch.float8_e4m3fn).double() * float(torch.tensor(scale))


class Exact:
    """The model's last layer and its scores in 64 bits, on the CPU."""

    def __init__(self, model, codes):
        self.model, self.codes, self.layer = model, codes, model.layers - 1
        self.token, self.position = model.token[-1].cpu(), model.position[-1].cpu()
        self.bigram, self.out = model.bigram.double().cpu(), model.out.double().cpu()

    def attention(self, tokens, seen=None):
        """Weights [Hq, keys], values [Hq, keys, dim] and O [Hq, dim] of the last token over all of them, or over what it is to see instead: (token, position) of each"""
        m, n = self.model, len(tokens)
        t, at = zip(*(list(zip(tokens, range(n))) if seen is None else seen))
        rows = lambda t, at: (self.token[torch.tensor(t)] + self.position[torch.tensor(at)]) * 0.7  # noqa: E731
        G, x = m.Hq // m.Hkv, rows(t, at)
        K, V = (through_the_cache(x[:, a:a + m.Hkv], self.codes).repeat_interleave(G, 1).transpose(0, 1) for a in (m.Hq, m.Hq + m.Hkv))
        w = torch.softmax((K @ rows(tokens[-1:], [n - 1])[0, :m.Hq].double()[:, :, None])[:, :, 0] / math.sqrt(m.dim), 1)
        return w, V, (w[:, :, None] * V).sum(1)

    def scores(self, token, O):
        return self.bigram[token] + O.flatten() @ self.out


def worst(exact, text):
    """The largest of (score of the best token - score of the one that was said) / what roundings may make of it; up to 1 the text is the model's"""
    m, most = exact.model, 0.0
    for n in range(1, len(text)):
        w, V, O = exact.attention(text[:n])
        scores = exact.scores(text[n - 1], O)
        best, said = int(scores.argmax()), text[n]
        if best == said:
            continue
        d = (exact.out[:, best] - exact.out[:, said]).view(m.Hq, m.dim)
        through = w * (V * d[:, None, :]).sum(2)
        sigma = 2 ** -8 / math.sqrt(3) * math.sqrt(float(((O * d) ** 2).sum() + (through ** 2).sum()))
        sums = 2 ** -12 * float(through.abs().sum()) + 2 ** -14 * float((O * d).abs().sum() + scores[best].abs() + scores[said].abs())
        most = max(most, float(scores[best] - scores[said]) / (SIGMAS * sigma + sums))
    return most


def wrong_texts(exact, what, count=5, steps=24):
    """Texts that the model would say if its attention were wrong: "parent" (the row before a token's own is not seen), "siblings" (two other tokens' rows at its own position are seen too), "none" (O is
    0), "rounded" (nothing is wrong but that O is bf16)"""
    out = []
    for b in range(count):
        text = [b]
        while len(text) < steps:
            n = len(text)
            seen = list(zip(text, range(n)))
            if what == "siblings":
                g = torch.Generator().manual_seed(100 * b + n)
                seen += [(t, n - 1) for t in torch.randint(0, exact.model.vocabulary, (2,), generator=g).tolist()]
            elif what == "parent" and n > 1:
                del seen[n - 2]
            O = exact.attention(text, seen)[2]
            O = O * 0 if what == "none" else O.to(torch.bfloat16).double() if what == "rounded" else O
            text.append(int(exact.scores(text[-1], O).argmax()))
        out.append(text)
    return out
