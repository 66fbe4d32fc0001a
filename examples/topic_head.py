#!/usr/bin/env python3
"""A head on a topic model: the sampler's topics as features for the next word.

    python examples/topic_head.py [--docs 400] [--vocab 3000] [--topics 64] [--width 256] [--steps 60]

Fits LDA to a synthetic corpus, takes every token's topic, and trains on the GPU

    embedding of the token's topic + embedding of the word before it
      -> layer norm (its input held in 8 bits for the backward pass)
      -> logits over the vocabulary -> softmax cross entropy with the token's word

with the operators of ``paper_1610_02496_amd.ops``.  Prints the training loss and, for documents that were left out of the
training, the loss next to that of the words' frequencies alone.
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

import corpusgen
import paper_1610_02496_amd as pk


class TopicHead(torch.nn.Module):
    """Scores words given the token's topic and the word before (index `vocab`: the document's start).  Parameters are
    float32; norm, logits and loss are computed in `dtype`."""

    def __init__(self, topics, vocab, width, dtype=torch.bfloat16):
        super().__init__()
        self.dtype = dtype
        self.topic = torch.nn.Parameter(torch.randn(topics, width) * 0.5)
        self.before = torch.nn.Parameter(torch.randn(vocab + 1, width) * 0.5)
        self.gain = torch.nn.Parameter(torch.ones(width))
        self.shift = torch.nn.Parameter(torch.zeros(width))
        self.words = torch.nn.Parameter(torch.randn(vocab, width) * width ** -0.5)

    def forward(self, topic, before, word, reduction="mean"):
        x = (self.topic[topic] + self.before[before]).to(self.dtype)
        y = pk.ops.layer_norm(x, self.gain, self.shift, checkpoint=True)
        return pk.ops.linear_cross_entropy(y, self.words.to(self.dtype), word, reduction)


def tokens(doc_ptr, word_ids, z, vocab):
    """(topic, word before, word) of every token, on the GPU."""
    before = np.empty_like(word_ids)
    before[1:] = word_ids[:-1]
    starts = doc_ptr[:-1][np.diff(doc_ptr) > 0]
    before[starts] = vocab
    return [torch.from_numpy(np.ascontiguousarray(a, dtype=np.int64)).cuda() for a in (z, before, word_ids)]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("docs", 400), ("vocab", 3000), ("topics", 64), ("width", 256), ("steps", 60), ("batch", 4096)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    torch.manual_seed(0)
    corpus = corpusgen.tiny(11, a.docs, a.vocab, 20, 120.0)
    with pk.Saber(corpus.doc_ptr, corpus.word_ids, a.vocab, a.topics, 50.0 / a.topics, 0.01, seed=1) as lda:
        lda.iterate(40)
        z = lda.get_z()
        print("LDA: %d tokens, log-likelihood %.4f per token" % (corpus.T, lda.loglik()))
    topic, before, word = tokens(corpus.doc_ptr, corpus.word_ids, z, a.vocab)
    split = int(corpus.doc_ptr[a.docs * 9 // 10])   # the last tenth of the documents is left out
    head = TopicHead(a.topics, a.vocab, a.width).cuda()
    step = torch.optim.Adam(head.parameters(), lr=0.01)
    losses = []
    for i in range(a.steps):
        pick = torch.randint(0, split, (min(a.batch, split),), device="cuda")
        loss = head(topic[pick], before[pick], word[pick])
        step.zero_grad(set_to_none=True)
        loss.backward()
        step.step()
        losses.append(loss.detach())
        if i % 10 == 0 or i == a.steps - 1:
            print("step %d: loss %.4f" % (i, float(losses[-1])))
    with torch.no_grad():
        held = float(head(topic[split:], before[split:], word[split:]))
        one = float(head(topic[split:split + 1], before[split:split + 1], word[split:split + 1]))   # a single token, as a server scores it
        count = torch.bincount(word[:split], minlength=a.vocab).double() + 0.01
        unigram = float(-(count / count.sum()).log()[word[split:]].mean())
    print("documents left out: loss %.4f, of the frequencies alone %.4f; their first token alone: %.4f" % (held, unigram, one))
    return [float(v) for v in losses], held, unigram, one


if __name__ == "__main__":
    main()
