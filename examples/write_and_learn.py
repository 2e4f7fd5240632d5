"""A model that writes, and a smaller one that learns from it: the operators beside the scoring step, run together.

    python examples/write_and_learn.py [--words 4000] [--hidden 128] [--sentences 64] [--length 24] [--passes 30]

A recurrent language model (random weights) takes one step per word for a batch of sentences: hidden update (rnnlm_step), whole rows
of logits from its output layer in 4 bits (rnnlm_q4_matvec), the next word (rnnlm_sample).  Its top logits at every step, and the word
it wrote, train the output layer of a student of a quarter of the hidden units (rnnlm_distill: loss and gradient in one call).  At
the end the student is loaded like any other model and scores held-out sentences with rnnlm_step.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2007_11794_amd as rn  # noqa: E402
from workloads import CONFIGS, make_model  # noqa: E402

DEV = "cuda:0"


class Writer:
    """A loaded model with its output layer in 4 bits, and the buffers of a batch of sentences, made once."""

    def __init__(self, weights, batch, group=64):
        self.V, self.H = weights["U"].shape
        self.batch = batch
        self.model = rn.rnnlm_load(self.V, self.H, rn.RNNLM_F32, weights["U"], weights["W"], weights["O"], weights["bias"], batch)
        codes, scales, zeros = rn.rnnlm_q4_quantize(weights["O"].T, group, zeros=True)
        self.group = group
        self.codes, self.scales, self.zeros = (torch.from_numpy(a).to(DEV) for a in (codes, scales, zeros))
        self.bias = torch.from_numpy(weights["bias"]).to(DEV)
        self.no_query, self.no_score = torch.empty((batch, 0), dtype=torch.int32, device=DEV), torch.empty((batch, 0), device=DEV)
        self.logits = torch.empty((batch, self.V), device=DEV)
        self.workspace = torch.empty(rn.rnnlm_sample_workspace_bytes(batch, self.V), dtype=torch.uint8, device=DEV)

    def hidden(self, word, h):
        out = torch.empty_like(h)
        rn.rnnlm_step(self.model, word, h, self.no_query, out, self.no_score)      # no words to score: the hidden vectors alone
        return out

    def write(self, length, generator, temperature=0.8, top_k=200, top_p=0.95, keep=32):
        """Sentences of `length` words: words int32 [length + 1, batch], log-probabilities [length, batch], and at every step the top
        `keep` logits, words int32 and values [length, batch, keep]."""
        N = self.batch
        limits = dict(temperature=torch.full((N,), temperature, device=DEV), top_k=torch.full((N,), top_k, dtype=torch.int32, device=DEV),
                      top_p=torch.full((N,), top_p, device=DEV))
        words, logprob = torch.zeros((length + 1, N), dtype=torch.int32, device=DEV), torch.empty((length, N), device=DEV)
        top_word, top_logit = torch.empty((length, N, keep), dtype=torch.int32, device=DEV), torch.empty((length, N, keep), device=DEV)
        h = torch.zeros((N, self.H), device=DEV)                                   # the start of a sentence
        for t in range(length):
            h = self.hidden(words[t], h)
            rn.rnnlm_q4_matvec(self.codes, self.scales, self.group, h, self.logits, zeros=self.zeros, bias=self.bias)
            u = torch.rand(N, generator=generator, device=DEV)
            rn.rnnlm_sample(self.logits, u, words[t + 1], logprob[t], self.workspace, **limits)
            value, word = self.logits.topk(keep, dim=1)
            top_logit[t], top_word[t] = value, word.int()
        return words, logprob, top_word, top_logit


def student_inputs(model, H, words):
    """The student's hidden vectors in front of every word: [length * batch, H]."""
    length, N = words.shape[0] - 1, words.shape[1]
    none, score = torch.empty((N, 0), dtype=torch.int32, device=DEV), torch.empty((N, 0), device=DEV)
    h, out = torch.zeros((N, H), device=DEV), torch.empty((length, N, H), device=DEV)
    for t in range(length):
        rn.rnnlm_step(model, words[t], h, none, out[t], score)
        h = out[t]
    return out.view(length * N, H)


def main(words=4000, hidden=128, sentences=64, length=24, passes=30, temperature=2.0, label_weight=0.25, seed=1):
    teacher_config = CONFIGS[2].scaled(V=words, H=hidden, sigma=0.3)
    teacher = make_model(teacher_config, seed=seed)
    teacher["bias"] = (-1.1 * np.log(np.arange(1, words + 1))).astype(np.float32)  # frequent words first
    writer = Writer(teacher, sentences)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    text, logprob, top_word, top_logit = writer.write(length, g)
    held_out = writer.write(length, g)[0]
    assert bool(((text >= 0) & (text < words)).all()) and bool(torch.isfinite(logprob).all())

    # The student: a quarter of the units, recurrent weights as they are drawn, its output layer to be learned.
    H = max(8, hidden // 4)
    small = make_model(teacher_config.scaled(H=H), seed=seed + 1)
    small["O"][:] = 0.0
    body = rn.rnnlm_load(words, H, rn.RNNLM_F32, small["U"], small["W"], small["O"], None, sentences)
    x = student_inputs(body, H, text)
    rows = x.shape[0]
    x1 = torch.cat([x - 0.5, torch.ones((rows, 1), device=DEV)], 1)                # with a column for the bias
    weights = torch.zeros((H + 1, words), device=DEV)
    moment, second = torch.zeros_like(weights), torch.zeros_like(weights)
    labels, top_word, top_logit = text[1:].reshape(rows).contiguous(), top_word.view(rows, -1), top_logit.view(rows, -1)
    loss, stats, grad = torch.empty(rows, device=DEV), torch.empty((rows, 4), device=DEV), torch.empty((rows, words), device=DEV)
    share = torch.full((rows,), 1.0 / rows, device=DEV)
    workspace = torch.empty(rn.rnnlm_distill_workspace_bytes(rows, words), dtype=torch.uint8, device=DEV)
    losses = []
    for step in range(1, passes + 1):
        logits = x1 @ weights
        rn.rnnlm_distill(logits, top_word, top_logit, loss, stats, workspace, temperature=temperature, labels=labels, label_weight=label_weight,
                         row_weight=share, grad=grad)
        losses.append(float(loss.mean()))
        d = x1.t() @ grad                                                          # Adam
        moment.lerp_(d, 0.1)
        second.lerp_(d * d, 0.01)
        weights -= 0.1 * (moment / (1 - 0.9 ** step)) / ((second / (1 - 0.99 ** step)).sqrt() + 1e-8)
    O = weights[:H].cpu().numpy()
    bias = (weights[H] - 0.5 * weights[:H].sum(0)).cpu().numpy()
    student = rn.rnnlm_load(words, H, rn.RNNLM_F32, small["U"], small["W"], np.ascontiguousarray(O), bias, sentences)

    def score(model, units):
        """Mean log-probability of the held-out sentences' words."""
        h, total = torch.zeros((sentences, units), device=DEV), 0.0
        for t in range(length):
            out, lp = torch.empty_like(h), torch.empty((sentences, 1), device=DEV)
            rn.rnnlm_step(model, held_out[t].contiguous(), h, held_out[t + 1].view(-1, 1).contiguous(), out, lp)
            h, total = out, total + float(lp.mean())
        return total / length

    result = {"losses": losses, "teacher": score(writer.model, hidden), "student": score(student, H), "untrained": score(body, H), "text": text.cpu().numpy()}
    for m in (student, body, writer.model):
        m.close()
    return result


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    for name, value in (("words", 4000), ("hidden", 128), ("sentences", 64), ("length", 24), ("passes", 30)):
        p.add_argument("--" + name, type=int, default=value)
    r = main(**vars(p.parse_args()))
    print("first sentence:", " ".join("w%d" % w for w in r["text"][:, 0]))
    print("loss: %.4f -> %.4f" % (r["losses"][0], r["losses"][-1]))
    print("log-probability of a held-out word: teacher %.3f, student %.3f, untrained %.3f" % (r["teacher"], r["student"], r["untrained"]))
