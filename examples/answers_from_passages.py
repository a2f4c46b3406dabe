"""Answers from retrieved passages: the index and a reader on one GPU.

    python examples/answers_from_passages.py

Passages are embedded (here: random vectors) into an index; each question's
nearest passages become a prompt, which goes through the attention layers of
a small random-weight language model with its keys and values kept in an 8-bit paged
cache; several answers are forked from each prompt and decoded a token at a
time, and the pages are given back.  It shows the calls in the order in which a
server makes them; the model has no trained weights and its answers no
meaning.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2607_16973_amd as tq  # noqa: E402


class Reader:
    """Attention layers with random weights: token embeddings, per layer a
    fused projection to queries, keys and values, and one back; logits."""

    def __init__(self, vocabulary=1000, layers=2, heads=8, kv_heads=2, head_dim=64, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.layers, self.heads, self.kv_heads, self.head_dim = layers, heads, kv_heads, head_dim
        width = heads * head_dim

        def weight(rows, columns):
            return (torch.randn(rows, columns, generator=g, device="cuda") / columns ** 0.5).to(torch.bfloat16)

        self.embedding = torch.randn(vocabulary, width, generator=g, device="cuda").to(torch.bfloat16)
        self.qkv = [weight(width + 2 * kv_heads * head_dim, width) for _ in range(layers)]
        self.back = [weight(width, width) for _ in range(layers)]
        self.logits = weight(vocabulary, width)

    def run(self, tokens, attend):
        """Logits of packed tokens; attend(layer, q, k, v) -> attention."""
        x = self.embedding[tokens]
        for layer in range(self.layers):
            y = torch.nn.functional.layer_norm(x.float(), x.shape[-1:]).to(x.dtype)
            qkv = (y @ self.qkv[layer].T).unflatten(1, (-1, self.head_dim))
            q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], 1)
            x = x + attend(layer, q, k, v).flatten(1) @ self.back[layer].T
        return x @ self.logits.T


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def answer(n_passages=2000, questions=3, top=4, answers=4, steps=12, kind="int8", seed=1):
    """Returns what each answer decoded ([questions * answers] lists), its logits at the last step, the whole
    token rows, the reader and the pages that are live at the end."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    reader = Reader(seed=seed)

    # the index: passages and their embeddings
    d = 256
    index = tq.Index(tq.Codebook(d, 4), tq.Rotation(d, seed))
    index.add(torch.randn(n_passages, d, generator=g, device="cuda"))
    lengths = torch.randint(20, 120, (n_passages,), generator=g, device="cuda")
    found, _ = index.search(torch.randn(questions, d, generator=g, device="cuda"), top)

    # one prompt per question: its passages' tokens, then the question's
    counts = (lengths[found].sum(1) + 9).tolist()
    tokens = torch.randint(0, len(reader.embedding), (sum(counts),), generator=g, device="cuda")
    starts = ints([0] + torch.tensor(counts).cumsum(0).tolist())

    # rows 0 .. questions - 1 hold the prompts, the answers follow
    rows = questions * (1 + answers)
    width = -(-(max(counts) + steps) // 64)
    cache = tq.KVCache(reader.layers, rows * width, reader.kv_heads, reader.head_dim, kind)
    pages = tq.KVPages(rows, width, rows * width)
    pages.resize(ints(counts + [0] * (rows - questions)), cache)

    def read_prompt(layer, q, k, v):
        cache.append(layer, k, v, pages.tables[:questions], pages.lens[:questions], starts)
        return tq.attention(q, k, v, starts, longest=max(counts))

    logits = reader.run(tokens, read_prompt)[starts[1:].long() - 1]

    # fork each prompt into its answers; they share its whole pages
    pages.fork(ints([q for q in range(questions) for _ in range(answers)]), ints(list(range(questions, rows))), cache)
    told = [[] for _ in range(questions * answers)]
    logits = logits.repeat_interleave(answers, 0)
    for step in range(steps):
        # each answer takes another of the likely tokens first, the likeliest afterwards
        best = logits.topk(answers, 1).indices
        pick = torch.arange(questions * answers, device="cuda") % answers if step == 0 else 0
        new = best[torch.arange(questions * answers, device="cuda"), pick]
        for row, token in zip(told, new.tolist()):
            row.append(token)
        goals = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
        goals[questions:] = pages.lens[questions:] + 1
        pages.resize(goals, cache)

        def decode(layer, q, k, v):
            cache.append(layer, k, v, pages.tables[questions:], pages.lens[questions:])
            return cache.attend(layer, q, pages.tables[questions:], pages.lens[questions:], longest=max(counts) + steps)

        logits = reader.run(new, decode)
    cache.check()

    # every other answer and the prompts are done: their pages go back, and the pool is closed up
    goals = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    goals[:questions] = 0
    goals[questions::2] = 0
    pages.resize(goals, cache)
    live = pages.compact(cache)
    cache.check()
    prompts = [tokens[a:b].tolist() for a, b in zip(starts[:-1].tolist(), starts[1:].tolist())]
    whole = [prompts[i // answers] + told[i] for i in range(questions * answers)]
    return told, logits, whole, reader, int(live.item())


def main():
    told, _, whole, _, live = answer()
    for i, row in enumerate(told):
        print("answer %2d (%4d tokens in all):" % (i, len(whole[i])), *row)
    print("%d pages stay in use" % live)


if __name__ == "__main__":
    main()
