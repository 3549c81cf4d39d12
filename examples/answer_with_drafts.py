"""Answers from retrieved passages with drafted tokens, over a quantised cache.

The passages of a micro-batch enter a cache of 8-bit numbers once and are the prefix that its queries share.  Then every step feeds each
query's last token and a few drafts: what followed the last place in passages, question and answer where that token stood.  One pass says what the
model makes of all of them, the drafts that it would have said itself are kept, and the lengths of the others are taken back: their
slots are written anew by the next step.  The steps are one graph.

The language model is a small decoder with random weights (that of answer_from_passages.py).

    python examples/answer_with_drafts.py
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import torch

import paper_2502_20969_amd as P
from answer_from_passages import D, HEADS, HIDDEN, LAYERS, PAGE, VOCAB, Model, i32


def caches(pages, quantised):
    def one():
        shape = (pages, PAGE, HEADS, D)
        if not quantised:
            return P.KvCache(*(torch.zeros(shape, dtype=torch.float16, device="cuda") for _ in range(2)))
        codes = (torch.zeros(shape, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
        powers = (torch.zeros(shape[:3], dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu) for _ in range(2))
        return P.KvCache(*codes, *powers, dtype=torch.float16)
    return [one() for _ in range(LAYERS)]


def answer(queries=3, drafts=4, new=40, passages=3, docs=400, dim=64, passage_tokens=60, question_tokens=9, quantised=True, graph=True, seed=0):
    """Returns the queries' answers (new tokens or a few more each), and how many steps they took."""
    g = torch.Generator().manual_seed(seed)
    vectors = torch.nn.functional.normalize(torch.randn(docs, dim, generator=g), dim=1)
    centroids = torch.nn.functional.normalize(torch.randn(16, dim, generator=g), dim=1)
    texts = torch.randint(1, VOCAB, (docs, passage_tokens), generator=g)
    asked = torch.nn.functional.normalize(vectors[torch.randint(0, docs, (1,), generator=g)] + 0.3 * torch.randn(queries, dim, generator=g) / dim ** 0.5, dim=1)
    questions = torch.randint(1, VOCAB, (queries, question_tokens), generator=g)
    index = P.ivf_build_layout(vectors, "f32", centroids, (vectors @ centroids.T).argmax(1).int(), metric=P.IVF_IP,
                               compute_stream=torch.cuda.Stream(), copy_stream=torch.cuda.Stream())
    ids, _ = index.ivf_search(asked.numpy(), 4, passages)
    index.close()
    prefix = torch.cat([texts[j] for j in sorted({int(j) for row in ids for j in row if j >= 0})])

    # pages: the passages', then each query's own
    fed = 1 + drafts
    room = question_tokens + new + 2 * fed
    shared, own = -(-len(prefix) // PAGE), -(-room // PAGE)
    layers = caches(shared + queries * own, quantised)
    model = Model(len(prefix) + room, seed)
    entries = i32(torch.arange(shared)[None])
    table = i32(shared + torch.arange(queries * own).view(queries, own))
    group = dict(group_off=i32([0, queries]), prefix_lens=i32([len(prefix)]), prefix_table=entries, max_prefix=len(prefix))
    fill = P.KvStep(i32([0, len(prefix)]), i32([len(prefix)]), entries, page=PAGE, n_tokens=len(prefix), max_q=len(prefix), max_len=len(prefix))
    model.step(prefix.cuda(), fill, layers)
    lens = i32([question_tokens] * queries)
    ask = P.KvStep(i32(torch.arange(queries + 1) * question_tokens), lens, table, page=PAGE, n_tokens=queries * question_tokens, max_q=question_tokens,
                   max_len=question_tokens, **group)
    hidden = model.step(questions.reshape(-1).cuda(), ask, layers).view(queries, question_tokens, HIDDEN)[:, -1]

    # what is known of each query's text: passages, question, answer
    known = torch.full((queries, len(prefix) + room), -2, dtype=torch.int32, device="cuda")
    begin = len(prefix) + question_tokens
    known[:, :begin] = torch.cat([prefix.expand(queries, -1), questions], 1).int().cuda()
    known[:, begin] = (hidden @ model.head).argmax(-1)
    upto = i32([begin + 1] * queries)                        # tokens that are known
    tokens = torch.full((queries, fed), -1, dtype=torch.int32, device="cuda")
    place = torch.arange(known.shape[1], device="cuda")
    ahead = torch.arange(fed, device="cuda")

    def look_up():
        """The last known token, and what followed it where it stood before; -1, which is refused, where nothing did."""
        last = known.gather(1, upto[:, None].long() - 1)
        seen = (known == last) & (place < upto[:, None] - 1)
        at = torch.where(seen, place, torch.full_like(place, -1)).amax(1, keepdim=True)
        from_ = at + ahead
        found = (at >= 0) & (from_ < upto[:, None])
        tokens.copy_(torch.where(found, known.gather(1, from_.clamp(0, known.shape[1] - 1)), torch.full_like(tokens, -1)))
        tokens[:, :1] = last

    step = P.KvStep(i32(torch.arange(queries + 1) * fed), lens, table, page=PAGE, n_tokens=queries * fed, max_q=fed, max_len=room, **group)

    def advance():
        look_up()
        lens.add_(fed)
        hidden = model.step(tokens.view(-1).clamp(min=0), step, layers)
        accepted, follows, _ = P.ivf_verify_draft(step, hidden @ model.head, tokens.view(-1), scale=0.0, lens_out=lens)
        said = torch.cat([tokens[:, 1:], follows[:, None]], 1)
        said = torch.where(ahead == accepted[:, None], follows[:, None], said)
        to = (upto[:, None] + ahead).long().clamp(max=known.shape[1] - 1)
        known.scatter_(1, to, torch.where(ahead <= accepted[:, None], said, torch.full_like(said, -2)))
        upto.add_(accepted + 1)
        # a query that has its answer waits for the others: its last tokens are said anew
        over = (upto - (begin + new)).clamp(min=0)
        upto.sub_(over)
        lens.sub_(over)

    steps, replay = 0, advance
    while int(upto.min()) < begin + new:
        if graph and steps == 2:                             # (after two by themselves, which let the libraries set up)
            recorded = torch.cuda.CUDAGraph()
            with torch.cuda.graph(recorded):
                advance()
            replay = recorded.replay
        replay()
        steps += 1
    return known[:, begin:begin + new].tolist(), steps


if __name__ == "__main__":
    for drafts in (0, 4):
        texts, steps = answer(drafts=drafts)
        print(f"{drafts} drafts a step: {steps} steps")
        for text in texts:
            print("  ", *text)
