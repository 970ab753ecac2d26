"""Greedy decoding with verified drafts on SBVR weights, all on the GPU.

A small randomly initialised decoder (grouped-query attention, gated MLP, norms
before and after each block) is quantised with the package's encoder and run
with its operators: a step plans its pages and masks (batch_plan), and per
layer takes norms (residual_norm), SBVR products, the cache write (cache_write)
and attention over the paged cache (tree_attention); adjust_logits applies the
request's penalty before the choice.

A draft proposes a tree of up to eight tokens: the last chosen token, and below
it guesses taken from where that token occurred before.  One step runs the whole
tree -- its tokens share the reading of the weights -- and every token whose
parent is accepted and chose it is accepted too.  The accepted tokens' keys and
values move to the front of the step's slots, and the next step continues there.

The verified tokens have to be those that single steps choose, up to the first
choice that rounding may turn: several tokens of a step run other products and
other attention kernels than one.  The program fails where they are not.

    python examples/verify_drafts.py [--tokens 64]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2509_18172_amd as sb  # noqa: E402

TREE = 8  # tokens of a step: what one small-batch product takes


class Decoder:
    """Weights, cache and step of the model."""

    def __init__(self, layers=2, width=512, heads=8, kv_heads=2, dim=64, inner=1024, vocab=1000, page_size=16,
                 pages=64, planes=4, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weight(out, inn):
            w = torch.randn(out, inn, generator=gen, device="cuda") * inn ** -0.5
            return sb.pack(*sb.encode(w, planes))

        def scale():
            return (1 + 0.1 * torch.randn(width, generator=gen, device="cuda")).half()
        self.heads, self.kv_heads, self.dim, self.width, self.vocab = heads, kv_heads, dim, width, vocab
        self.embedding = torch.randn(vocab, width, generator=gen, device="cuda").half()
        self.layers = [dict(qkv=weight((heads + 2 * kv_heads) * dim, width), o=weight(width, heads * dim),
                            gate_up=weight(2 * inner, width), down=weight(width, inner),
                            cache=sb.KVCache.alloc(pages, page_size, kv_heads, dim),
                            norms=[scale() for _ in range(4)]) for _ in range(layers)]
        self.last_norm, self.head = scale(), weight(vocab, width)
        # each of the 2 blocks a layer adds its share of the final stream
        self.block_scale = (2 * layers) ** -0.5
        self.free = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
        self.table = torch.full((1, pages), -1, dtype=torch.int32, device="cuda")
        self.page_size, self.taken, self.context = page_size, 0, 0
        self.frequency = 10000.0 ** (-torch.arange(0, dim, 2, device="cuda") / dim)

    @staticmethod
    def product(weight, x):
        return sb.gemm_small_batch(weight, x) if x.shape[0] <= 8 else sb.gemm_prefill(weight, x)

    def rotate(self, x, positions):
        angle = positions[:, None].float() * self.frequency
        cos, sin = angle.cos()[:, None], angle.sin()[:, None]
        a, b = x.float().chunk(2, dim=-1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1).half()

    def step(self, tokens, parents=None):
        """Logits [tokens][vocab] (binary32) of a chain of up to 64 tokens, or
        of a tree with the given parents, after the context."""
        T = len(tokens)
        ids = torch.tensor(tokens, device="cuda")
        lens = torch.tensor([self.context], dtype=torch.int32, device="cuda")
        new = torch.tensor([T], dtype=torch.int32, device="cuda")
        if parents is not None:
            parents = torch.tensor(parents, dtype=torch.int32, device="cuda")
        plan = sb.batch_plan(lens, new, self.free[self.taken:], self.table, self.page_size, T, parents=parents)
        self.taken += -(-(self.context + T) // self.page_size) - -(-self.context // self.page_size)
        H, K, D = self.heads, self.kv_heads, self.dim
        x, y, post = self.embedding[ids].float(), None, None
        for layer in self.layers:
            pre_attn, post_attn, pre_mlp, post_mlp = layer["norms"]
            x, h = sb.residual_norm(x, y, post_weight=post, scale=self.block_scale, pre_weight=pre_attn)
            qkv = self.product(layer["qkv"], h).view(T, H + 2 * K, D)
            q, k = self.rotate(qkv[:, :H], plan.positions), self.rotate(qkv[:, H:H + K], plan.positions)
            sb.cache_write(layer["cache"], k, qkv[:, H + K:], plan.slots)
            a = sb.tree_attention(q, layer["cache"], self.table, lens, plan.query_start, plan.tree_mask, max_new=T)
            y = self.product(layer["o"], a.view(T, H * D))
            x, h = sb.residual_norm(x, y, post_weight=post_attn, scale=self.block_scale, pre_weight=pre_mlp)
            gate, up = self.product(layer["gate_up"], h).float().chunk(2, dim=1)
            y, post = self.product(layer["down"], (torch.nn.functional.silu(gate) * up).half()), post_mlp
        x, h = sb.residual_norm(x, y, post_weight=post, scale=self.block_scale, pre_weight=self.last_norm)
        self.plan = plan
        return self.product(self.head, h)

    def keep(self, accepted):
        """Makes the given tokens of the last step, a path from its root, the
        context's continuation: their keys and values move together."""
        index = torch.tensor(accepted, device="cuda")
        old, new = self.plan.slots[index], self.plan.slots[:len(accepted)].contiguous()
        at = old // self.page_size, old % self.page_size
        for layer in self.layers:
            cache = layer["cache"]
            sb.cache_write(cache, cache.k[at], cache.v[at], new)
        last = self.context + self.plan.slots.shape[0]
        self.context += len(accepted)
        # pages past the kept tokens go back to the front of the free list
        held, got = -(-self.context // self.page_size), -(-last // self.page_size)
        self.taken -= got - held


def draft(text):
    """A tree below the last token: tokens and their parents.  The guesses
    continue its latest occurrences, three tokens deep where there is room."""
    tokens, parents, seen = [text[-1]], [-1], set()
    for i in range(len(text) - 2, -1, -1):
        if text[i] != text[-1]:
            continue
        at, path = 0, ()
        for token in text[i + 1:i + 4]:
            path += (token,)
            if path in seen:
                at = next(j for j in range(1, len(tokens)) if parents[j] == at and tokens[j] == token)
                continue
            if len(tokens) == TREE:
                return tokens, parents
            seen.add(path)
            tokens.append(token)
            parents.append(at)
            at = len(tokens) - 1
    return tokens, parents


# Leads over the second choice, in parts of the largest logit, that rounding may
# turn: some two dozen binary16 roundings of 2^-11 lie between the runs, behind norms
# that may stretch them a few times, 2e-2 of the largest logit for each of the two.
NEAR = 4e-2


def generate(model, prompt, n, verify, repetition=1.05, propose=draft, leads=None):
    """n greedy tokens after the prompt: (tokens, steps taken).  propose: the
    tree for a text; leads: a list that gets each token's lead."""
    text, steps = list(prompt), 0
    for i in range(0, len(prompt) - 1, 64):
        chunk = prompt[i:min(i + 64, len(prompt) - 1)]
        model.step(chunk)
        model.keep(list(range(len(chunk))))
    penalty = torch.tensor([repetition], device="cuda")
    while len(text) < len(prompt) + n:
        tokens, parents = propose(text) if verify else (text[-1:], [-1])
        logits = model.step(tokens, parents)
        past = torch.tensor(text[:-1], dtype=torch.int32, device="cuda")  # the last one is the tree's root
        plan, T = model.plan, len(tokens)
        logits = sb.adjust_logits(logits, history=past, prompt_lens=torch.tensor([len(prompt)], dtype=torch.int32, device="cuda"),
                                  history_start=torch.tensor([0, len(text) - 1], dtype=torch.int32, device="cuda"),
                                  repetition=penalty, token_request=plan.token_request, query_start=plan.query_start,
                                  tree_mask=plan.tree_mask, draft_tokens=torch.tensor(tokens, dtype=torch.int32, device="cuda"),
                                  out_dtype=torch.float32)
        choice = logits.argmax(dim=1).tolist()
        if leads is not None:
            best = logits.topk(2, dim=1).values
            lead = ((best[:, 0] - best[:, 1]) / logits.abs().amax(dim=1)).tolist()
        accepted = [0]
        while True:
            text.append(choice[accepted[-1]])
            if leads is not None:
                leads.append(lead[accepted[-1]])
            child = next((j for j in range(T) if parents[j] == accepted[-1] and tokens[j] == text[-1]), None)
            if child is None:
                break
            accepted.append(child)
        model.keep(accepted)
        steps += 1
    return text[len(prompt):len(prompt) + n], steps


def first_difference(plain, verified):
    """The number of tokens that both have from the start."""
    return next((i for i, (a, b) in enumerate(zip(plain, verified)) if a != b), min(len(plain), len(verified)))


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=64)
    args = ap.parse_args()
    prompt = torch.randint(0, 1000, (100,), generator=torch.Generator().manual_seed(1)).tolist() * 2
    leads = []
    plain, steps = generate(Decoder(), prompt, args.tokens, verify=False, leads=leads)
    print(f"plain:    {args.tokens} tokens in {steps} steps")
    verified, steps = generate(Decoder(), prompt, args.tokens, verify=True)
    same = first_difference(plain, verified)
    print(f"verified: {args.tokens} tokens in {steps} steps, the first {same} the plain run's")
    if same < args.tokens:
        print(f"token {same} led by {leads[same]:.4f} of the largest logit; rounding may turn {NEAR}")
        if leads[same] > NEAR:
            sys.exit("verified decoding is not plain decoding")


if __name__ == "__main__":
    main()
