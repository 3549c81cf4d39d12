"""Answers from retrieved passages: scheduling, search, a shared paged cache and a beam search in one program.

Queries are put into micro-batches by the clusters that they probe, and searched.  The passages of a micro-batch enter the cache
once and are the prefix that its queries share; each question follows in slots of its own; then every step appends one
token per beam, attends over passages, question and answer so far, and picks the beams' continuations.  A beam's past
is its row of the table: it is moved by that row alone, and no key or value is copied.

The language model is a small decoder with random weights: attention, cache and selection are the library's, the products with
weights are torch's.

    python examples/answer_from_passages.py
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2502_20969_amd as P

HIDDEN, LAYERS, Q_HEADS, HEADS, D, VOCAB, PAGE = 256, 2, 8, 2, 64, 1000, 16
EOS = 0


class Model:
    def __init__(self, positions, seed=0):
        g = torch.Generator().manual_seed(seed)
        w = lambda *shape: (torch.randn(*shape, generator=g) / shape[0] ** 0.5).cuda()
        self.embed = torch.randn(VOCAB, HIDDEN, generator=g).cuda()
        self.head = w(HIDDEN, VOCAB) * 2
        self.layers = [dict(q=w(HIDDEN, Q_HEADS * D), k=w(HIDDEN, HEADS * D), v=w(HIDDEN, HEADS * D), o=w(Q_HEADS * D, HIDDEN),
                            up=w(HIDDEN, 2 * HIDDEN), down=w(2 * HIDDEN, HIDDEN)) for _ in range(LAYERS)]
        angle = torch.arange(positions)[:, None] * 10000.0 ** (-torch.arange(D // 2) * 2 / D)[None]
        self.rotary = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()

    @staticmethod
    def norm(x):
        return x * (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt()

    def run(self, tokens, attention):
        """Hidden states of `tokens`; attention(layer, q, k, v) sees the unrotated rows of every token."""
        x = self.embed[tokens]
        for i, w in enumerate(self.layers):
            h = self.norm(x)
            y = attention(i, (h @ w["q"]).view(-1, Q_HEADS, D), (h @ w["k"]).view(-1, HEADS, D), (h @ w["v"]).view(-1, HEADS, D))
            x = x + y.reshape(-1, Q_HEADS * D).float() @ w["o"]
            x = x + torch.relu(self.norm(x) @ w["up"]) @ w["down"]
        return self.norm(x)

    def step(self, tokens, step, caches):
        """The new tokens of a step, through the paged caches."""
        def attention(i, q, k, v):
            q, k, v = q.half(), k.half(), v.half()
            P.ivf_kv_append(step, caches[i], k, v, rotary=self.rotary, q=q, q_out=q)
            return P.ivf_attend(step, caches[i], q)
        return self.run(tokens, attention)

    def plain(self, tokens):
        """The same without a cache, in 32 bits: logarithms of the probabilities after every token."""
        n = tokens.shape[0]
        c, s = self.rotary[:n, None, :D // 2], self.rotary[:n, None, D // 2:]

        def turn(x):
            a, b = x[..., :D // 2], x[..., D // 2:]
            return torch.cat([a * c - b * s, b * c + a * s], -1)

        def attention(i, q, k, v):
            q, k, v = turn(q).transpose(0, 1), turn(k).repeat_interleave(Q_HEADS // HEADS, 1).transpose(0, 1), v.repeat_interleave(Q_HEADS // HEADS, 1).transpose(0, 1)
            x = (q.contiguous() @ k.transpose(1, 2).contiguous()) * D ** -0.5
            x = x.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -float("inf"))
            return (x.softmax(-1) @ v.contiguous()).transpose(0, 1)
        return (self.run(tokens, attention) @ self.head).log_softmax(-1)


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


def answer(queries=6, micro=3, beams=4, new=10, passages=3, docs=400, dim=64, passage_tokens=120, question_tokens=9, seed=0):
    """Returns the model and, per query, (the tokens it was asked with, [(score, answer)] best first)."""
    g = torch.Generator().manual_seed(seed)
    vectors = torch.nn.functional.normalize(torch.randn(docs, dim, generator=g), dim=1)
    centroids = torch.nn.functional.normalize(torch.randn(16, dim, generator=g), dim=1)
    texts = torch.randint(1, VOCAB, (docs, passage_tokens), generator=g)
    asked = torch.nn.functional.normalize(vectors[torch.randint(0, docs, (queries,), generator=g)] + 0.3 * torch.randn(queries, dim, generator=g), dim=1)
    questions = torch.randint(1, VOCAB, (queries, question_tokens), generator=g)

    # retrieval: micro-batches of queries that probe the same clusters, and their passages
    index = P.ivf_build_layout(vectors, "f32", centroids, (vectors @ centroids.T).argmax(1).int(), metric=P.IVF_IP,
                               compute_stream=torch.cuda.Stream(), copy_stream=torch.cuda.Stream())
    order = index.ivf_schedule(asked.numpy(), micro).tolist()
    ids, _ = index.ivf_search(asked.numpy(), 4, passages)
    index.close()
    batches = [order[i:i + micro] for i in range(0, queries, micro)]
    order = [q for batch in batches for q in batch]
    prefixes = [torch.cat([texts[j] for j in sorted({int(j) for q in batch for j in ids[q] if j >= 0})]) for batch in batches]

    # slots: whole pages for a prefix, single ones for everything else
    rows, lens = queries * beams, [len(p) for p in prefixes]
    pages = [(n + PAGE - 1) // PAGE for n in lens]
    first = sum(pages) * PAGE                                # the questions' slots, then one per beam and step
    n_pages = (first + queries * question_tokens + rows * new + PAGE - 1) // PAGE
    caches = [P.KvCache(*(torch.empty(n_pages, PAGE, HEADS, D, dtype=torch.float16, device="cuda") for _ in range(2))) for _ in range(LAYERS)]
    model = Model(max(lens) + question_tokens + new, seed)
    entries = torch.zeros(len(batches), max(pages), dtype=torch.int32)
    for b, n in enumerate(pages):
        entries[b, :n] = torch.arange(n) + sum(pages[:b])
    entries, prefix_lens, starts = entries.cuda(), i32(lens), [0]
    for batch in batches:
        starts.append(starts[-1] + len(batch))

    # the passages of every micro-batch, once
    offsets = i32([0] + torch.tensor(lens).cumsum(0).tolist())
    fill = P.KvStep(offsets, prefix_lens, entries, page=PAGE, n_tokens=sum(lens), max_q=max(lens), max_len=max(lens))
    model.step(torch.cat(prefixes).cuda(), fill, caches)

    # the questions behind them; a beam's table row names the slots of its question and of its answer
    shared = dict(prefix_lens=prefix_lens, prefix_table=entries, prefix_page=PAGE, max_prefix=max(lens))
    table = torch.zeros(queries, question_tokens + new, dtype=torch.int32)
    table[:, :question_tokens] = first + torch.arange(queries * question_tokens).view(queries, -1)
    table = table.cuda()
    ask = P.KvStep(i32(torch.arange(queries + 1) * question_tokens), i32([question_tokens] * queries), table, page=1, n_tokens=queries * question_tokens,
                   max_q=question_tokens, max_len=question_tokens, group_off=i32(starts), **shared)
    hidden = model.step(questions[order].reshape(-1).cuda(), ask, caches).view(queries, question_tokens, HIDDEN)[:, -1]

    # the first tokens: one beam a query becomes several
    tables = [torch.zeros(rows, question_tokens + new, dtype=torch.int32, device="cuda") for _ in range(2)]
    texts_of = [torch.full((rows, new), EOS, dtype=torch.int32, device="cuda") for _ in range(2)]
    start = torch.full((queries, new), EOS, dtype=torch.int32, device="cuda")
    score, _, token, done = P.ivf_beam_step((hidden @ model.head).view(queries, 1, VOCAB), torch.zeros(queries, 1, device="cuda"), beams,
                                            eos=EOS, states=[(table, tables[0]), (start, texts_of[0])])
    texts_of[0][:, 0] = token.view(-1)
    own = i32([question_tokens] * rows)
    steps = [P.KvStep(i32(torch.arange(rows + 1)), own, t, page=1, n_tokens=rows, max_q=1, max_len=question_tokens + new,
                      group_off=i32([s * beams for s in starts]), **shared) for t in tables]
    slots = i32(first + queries * question_tokens + torch.arange(rows))
    at = 0                                                   # the tables in use
    for n in range(1, new):
        tables[at].scatter_(1, own[:, None].long(), (slots + (n - 1) * rows)[:, None])
        own += 1
        hidden = model.step(token.view(-1).clamp(min=0), steps[at], caches)
        score, _, token, done = P.ivf_beam_step((hidden @ model.head).view(queries, beams, VOCAB), score, done=done, eos=EOS,
                                                states=[(tables[at], tables[1 - at]), (texts_of[at], texts_of[1 - at])])
        at = 1 - at
        texts_of[at][:, n] = token.view(-1)
    out = [None] * queries
    for i, q in enumerate(order):
        b = next(b for b, batch in enumerate(batches) if q in batch)
        found = [(float(score[i, j]), texts_of[at][i * beams + j].tolist()) for j in range(beams)]
        out[q] = (torch.cat([prefixes[b], questions[q]]), found)
    return model, out


def plain_score(model, prompt, text):
    """The score of an answer, by the whole sequence at once."""
    if EOS in text:
        text = text[:text.index(EOS) + 1]
    logp = model.plain(torch.cat([prompt, torch.tensor(text)]).cuda())
    return float(sum(logp[len(prompt) - 1 + i, t] for i, t in enumerate(text)))


if __name__ == "__main__":
    model, answers = answer()
    for q, (prompt, found) in enumerate(answers):
        print(f"query {q}: {len(prompt)} tokens of passages and question")
        for score, text in found:
            print(f"  {score:9.4f}  (computed plainly {plain_score(model, prompt, text):9.4f})  {text}")
