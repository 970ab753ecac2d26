"""The example that runs the operators of a step together: a drafted tree
gives the logits that its tokens give one by one, and verified decoding
continues where plain decoding does."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("verify_drafts", os.path.join(ROOT, "examples", "verify_drafts.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_a_tree_gives_the_logits_of_its_paths(example):
    prompt = torch.randint(0, 1000, (70,), generator=torch.Generator().manual_seed(3)).tolist()
    tokens, parents = [5, 17, 300, 42, 8, 999], [-1, 0, 0, 1, 2, 3]
    tree = example.Decoder(seed=1)
    for i in (0, 64):
        tree.step(prompt[i:i + 64])
        tree.keep(list(range(len(prompt[i:i + 64]))))
    got = tree.step(tokens, parents).double()
    for node in range(len(tokens)):
        path, up = [], node
        while up >= 0:
            path.insert(0, tokens[up])
            up = parents[up]
        chain = example.Decoder(seed=1)
        for i in (0, 64):
            chain.step(prompt[i:i + 64])
            chain.keep(list(range(len(prompt[i:i + 64]))))
        for token in path:
            want = chain.step([token])[0].double()
            chain.keep([0])
        # about two dozen binary16 roundings of 2^-11 between the two, behind
        # norms that may stretch them a few times
        assert float((got[node] - want).abs().max()) <= 2e-2 * float(want.abs().max()), node


def test_accepted_tokens_are_kept_in_place(example):
    """After a branch is accepted, the next step sees exactly its path."""
    prompt = list(range(100, 130))
    a, b = example.Decoder(seed=2), example.Decoder(seed=2)
    for m in (a, b):
        m.step(prompt)
        m.keep(list(range(len(prompt))))
    a.step([1, 2, 3, 4, 5, 6, 7], [-1, 0, 0, 2, 3, 0, 4])
    a.keep([0, 2, 3, 4])
    for token in (1, 3, 4, 5):
        b.step([token])
        b.keep([0])
    assert a.context == b.context == len(prompt) + 4
    x, y = a.step([50])[0].double(), b.step([50])[0].double()
    assert float((x - y).abs().max()) <= 2e-2 * float(y.abs().max())


def test_generation(example):
    prompt = torch.randint(0, 1000, (40,), generator=torch.Generator().manual_seed(5)).tolist() * 2
    plain, steps = example.generate(example.Decoder(), prompt, 24, verify=False)
    assert steps == 24 and len(plain) == 24
    verified, fewer = example.generate(example.Decoder(), prompt, 24, verify=True)
    assert len(verified) == 24 and fewer <= 24
    assert verified[0] == plain[0]


@pytest.mark.parametrize("seed", [0, 1, 2])
def test_verified_tokens_are_the_plain_ones(example, seed):
    """With drafts that hold the plain run's next three tokens, each beside a
    wrong one, every step takes four tokens, up to the first choice that
    rounding may turn; and the tokens are the plain run's."""
    n, prompt = 40, torch.randint(0, 1000, (50,), generator=torch.Generator().manual_seed(seed)).tolist()
    leads = []
    plain, _ = example.generate(example.Decoder(seed=seed), prompt, n + 4, verify=False, leads=leads)
    known = prompt + plain
    assert len(plain) == n + 4 and len(leads) == n + 4

    def propose(text):
        tokens, parents, at = [text[-1]], [-1], 0
        for token in known[len(text):len(text) + 3]:
            tokens += [(token + 1) % 1000, token]
            parents += [at, at]
            at = len(tokens) - 1
        return tokens + [(known[min(len(text) + 3, len(known) - 1)] + 1) % 1000], parents + [at]
    verified, steps = example.generate(example.Decoder(seed=seed), prompt, n, verify=True, propose=propose)
    same = example.first_difference(plain[:n], verified)
    assert same == n or leads[same] <= example.NEAR, (same, leads[same])
    assert same >= 4 and steps <= -(-same // 4) + n - same, (steps, same)


def test_the_program_fails_where_tokens_differ(example, monkeypatch):
    """A step that keeps the wrong tokens is found."""
    monkeypatch.setattr("sys.argv", ["verify_drafts.py", "--tokens", "24"])
    example.main()
    generate, changed = example.generate, []

    def spoilt(model, prompt, n, verify, **more):
        tokens, steps = generate(model, prompt, n, verify, **more)
        if verify:
            tokens[changed[0]] = (tokens[changed[0]] + 1) % 1000
        else:
            changed.append(max(range(n), key=lambda i: more["leads"][i]))
        return tokens, steps
    monkeypatch.setattr(example, "generate", spoilt)
    with pytest.raises(SystemExit):
        example.main()
