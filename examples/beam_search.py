"""Beam search on SBVR weights, all on the GPU: the host never waits for a step.

The small decoder of verify_drafts.py, with the rotation of queries and keys in the
pass that writes the cache (rotary_write).  A request's beams are rows of one page
table.  A step asks which pages are free (page_usage), plans (batch_plan), runs the
layers, chooses the continuations (beam_select) and makes the next rows from their
parents: they share all full pages, and the partly filled one is copied (page_fork,
page_copy).  Now and then the pages are moved together (page_compact).

The search is run a second time with every row's pages its own, copied whole at each
step.  Both take the same products and the same attention, so their tokens and scores
have to be the same, bit for bit; the program fails where they are not.

    python examples/beam_search.py [--tokens 40] [--beams 4]
"""
import argparse
import os
import sys

import torch

sys.path[:0] = [os.path.dirname(os.path.dirname(os.path.abspath(__file__))), os.path.dirname(os.path.abspath(__file__))]
import paper_2509_18172_amd as sb  # noqa: E402
from verify_drafts import Decoder  # noqa: E402


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def forward(model, tokens, plan, lens, table, max_new):
    """Logits [tokens][vocab] of a planned step of the decoder."""
    H, K, D, T = model.heads, model.kv_heads, model.dim, tokens.shape[0]
    x, y, post = model.embedding[tokens.long()].float(), None, None
    for layer in model.layers:
        pre_attn, post_attn, pre_mlp, post_mlp = layer["norms"]
        x, h = sb.residual_norm(x, y, post_weight=post, scale=model.block_scale, pre_weight=pre_attn)
        qkv = model.product(layer["qkv"], h).view(T, H + 2 * K, D)
        q = sb.rotary_write(qkv[:, :H], layer["cache"], qkv[:, H:H + K], qkv[:, H + K:], plan.slots, plan.positions,
                            model.frequency)
        a = sb.tree_attention(q, layer["cache"], table, lens, plan.query_start, plan.tree_mask, max_new=max_new)
        y = model.product(layer["o"], a.view(T, H * D))
        x, h = sb.residual_norm(x, y, post_weight=post_attn, scale=model.block_scale, pre_weight=pre_mlp)
        gate, up = model.product(layer["gate_up"], h).float().chunk(2, dim=1)
        y, post = model.product(layer["down"], (torch.nn.functional.silu(gate) * up).half()), post_mlp
    return model.product(model.head, sb.residual_norm(x, y, post_weight=post, scale=model.block_scale,
                                                      pre_weight=model.last_norm)[1])


class SharedPages:
    """Rows that share pages.  compact_every: the steps after which the pages are
    moved together."""

    def __init__(self, model, rows, width, compact_every=8):
        self.caches, self.page_size = [layer["cache"] for layer in model.layers], model.page_size
        self.pages = self.caches[0].k.shape[0]
        self.lens, self.table = ints([0] * rows), torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
        self.steps, self.compact_every = 0, compact_every

    def plan(self, new, tokens):
        self.usage = sb.page_usage(self.lens, self.table, self.page_size, self.pages)
        self.now = sb.batch_plan(self.lens, new, self.usage.free_pages, self.table, self.page_size, tokens)
        return self.now

    def follow(self, parents):
        """The rows whose parents these are (int32 [requests][beams], within each
        request) instead of the present ones."""
        f = sb.page_fork(self.lens, self.table, parents, self.page_size, self.usage.free_pages, taken=self.now.used)
        sb.page_copy(self.caches, f.src, f.dst, f.tokens)
        self.lens, self.table = f.context_lens, f.page_table
        self.steps += 1
        if self.steps % self.compact_every == 0:
            moved = sb.page_compact(self.lens, self.table, self.page_size, self.pages)
            sb.page_copy(self.caches, moved.src, moved.dst)
            self.table = moved.page_table


class OwnPages:
    """Rows with pages of their own, copied whole."""

    def __init__(self, model, rows, width):
        self.caches, self.page_size, self.width = [layer["cache"] for layer in model.layers], model.page_size, width
        self.set_rows(rows)
        self.lens = ints([0] * rows)

    def set_rows(self, rows):
        self.table = torch.arange(rows * self.width, dtype=torch.int32, device="cuda").view(rows, self.width)

    def plan(self, new, tokens):
        plan = sb.batch_plan(self.lens, new, self.table.view(-1), self.table.clone(), self.page_size, tokens)
        row = plan.token_request.long()
        at = self.lens[row].long() + torch.arange(tokens, device="cuda") - plan.query_start.long()[row]
        plan.slots = self.table[row, at // self.page_size] * self.page_size + at % self.page_size
        return plan

    def follow(self, parents):
        requests, beams = parents.shape
        per = self.lens.shape[0] // requests
        row = (torch.arange(requests, device="cuda")[:, None] * per + parents).view(-1)
        pages = self.table[row].long()
        self.lens = self.lens[row]
        self.set_rows(requests * beams)
        for cache in self.caches:
            for t in (cache.k, cache.v):
                t[self.table.long()] = t[pages]


def search(model, prompts, beams, n, end, store=SharedPages, **more):
    """n steps of beam search after the prompts, without waiting for the GPU.
    Returns the beams' tokens [requests][beams][n] and scores [requests][beams], and
    per step what ended: scores and tokens so far."""
    requests = len(prompts)
    width = (max(map(len, prompts)) + n) // model.page_size + 2
    store = store(model, requests, width, **more)
    # the prompts but for their last tokens, up to 64 tokens of each at a time
    for i in range(0, max(len(p) for p in prompts) - 1, 64):
        chunks = [p[:-1][i:i + 64] for p in prompts]
        new = ints([len(c) for c in chunks])
        tokens = ints(sum(chunks, []))
        plan = store.plan(new, tokens.shape[0])
        forward(model, tokens, plan, store.lens, store.table, 64)
        store.lens = store.lens + new
    tokens = ints([p[-1] for p in prompts])
    scores = torch.zeros(requests, 1, device="cuda")
    history = torch.empty(requests, 1, 0, dtype=torch.int32, device="cuda")
    ends, ended = ints([end]), []
    for _ in range(n):
        rows = tokens.numel()
        new = torch.ones(rows, dtype=torch.int32, device="cuda")
        plan = store.plan(new, rows)
        logits = forward(model, tokens.view(-1), plan, store.lens, store.table, 1)
        choice = sb.beam_select(logits, scores, n=beams, end_tokens=ends)
        ended.append((choice.ended, history))
        store.lens = store.lens + new
        store.follow(choice.parents)
        # (a row that found no continuation has the parent -1 and the score -infinity; its history is not used)
        parents = choice.parents.long().clamp(min=0)
        kept = history.gather(1, parents[:, :, None].expand(-1, -1, history.shape[2]))
        history = torch.cat([kept, choice.tokens[:, :, None]], dim=2)
        tokens, scores = choice.tokens, choice.scores
    return history, scores, ended


def best(history, scores, ended, length_penalty=1.0):
    """The best hypothesis of each request, those that ended and those that go on:
    (score by length, tokens)."""
    found = []
    for r in range(history.shape[0]):
        every = [(s / len(h) ** length_penalty, h) for s, h in zip(scores[r].tolist(), history[r].tolist())]
        for step_scores, step_history in ended:
            every += [(s / (len(h) + 1) ** length_penalty, h)
                      for s, h in zip(step_scores[r].tolist(), step_history[r].tolist()) if s > -float("inf")]
        found.append(max(every))
    return found


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=40)
    ap.add_argument("--beams", type=int, default=4)
    args = ap.parse_args()
    gen = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, 1000, (length,), generator=gen).tolist() for length in (75, 20)]
    runs = [search(Decoder(pages=256), prompts, args.beams, args.tokens, end=7, store=store)
            for store in (SharedPages, OwnPages)]
    for r, (score, tokens) in enumerate(best(*runs[0])):
        print(f"request {r}: {score:.4f} a token, {len(tokens)} tokens, {tokens[:8]} ...")
    if not all(torch.equal(a, b) for a, b in zip(runs[0][:2], runs[1][:2])):
        sys.exit("the search on shared pages is not the one on pages of each row's own")
    print("shared pages and pages of each row's own: the same tokens and scores")


if __name__ == "__main__":
    main()
