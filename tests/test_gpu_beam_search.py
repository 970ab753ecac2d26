"""The example that runs the operators of a beam search together: on shared pages it
is the search on pages of each row's own, and its scores are those of its tokens."""
import importlib.util
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    spec = importlib.util.spec_from_file_location("beam_search", os.path.join(ROOT, "examples", "beam_search.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def prompts(*lengths):
    gen = torch.Generator().manual_seed(sum(lengths))
    return [torch.randint(0, 1000, (n,), generator=gen).tolist() for n in lengths]


@pytest.mark.parametrize("lengths,beams,n,page,every", [((75, 20), 4, 40, 16, 8), ((1,), 8, 20, 16, 1), ((17, 33, 2, 5), 2, 35, 32, 3),
                                                        ((130,), 1, 5, 16, 2)])
def test_shared_pages_change_nothing(example, lengths, beams, n, page, every):
    runs = []
    for store, more in ((example.SharedPages, dict(compact_every=every)), (example.OwnPages, {})):
        model = example.Decoder(pages=256, page_size=page, seed=2)
        runs.append(example.search(model, prompts(*lengths), beams, n, end=7, store=store, **more))
    (tokens, scores, ended), (want_tokens, want_scores, want_ended) = runs
    assert torch.equal(tokens, want_tokens) and torch.equal(scores, want_scores)
    assert all(torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) for a, b in zip(ended, want_ended))
    assert bool((tokens >= 0).all()) and bool((scores[:, :-1] >= scores[:, 1:]).all())


def test_fewer_continuations_than_beams(example, monkeypatch):
    """Two tokens allowed and four beams: two rows of the first step have no parent, and
    the second step fills them."""
    plain, allowed = example.forward, [3, 500]

    def masked(*args):
        logits = plain(*args).float()
        only = torch.full_like(logits, -float("inf"))
        only[:, allowed] = logits[:, allowed]
        return only
    monkeypatch.setattr(example, "forward", masked)
    for n in (1, 2, 6):
        runs = [example.search(example.Decoder(pages=256, seed=4), prompts(20, 33), 4, n, end=7, store=store)
                for store in (example.SharedPages, example.OwnPages)]
        (tokens, scores, _), (want_tokens, want_scores, _) = runs
        assert torch.equal(tokens, want_tokens) and torch.equal(scores, want_scores)
        assert scores.isfinite().sum(1).tolist() == [min(2 ** n, 4)] * 2
        assert set(tokens[scores.isfinite()].flatten().tolist()) <= set(allowed)


def test_scores_are_the_tokens_own(example):
    """A beam's score is the sum of its tokens' log probabilities, as plain steps on
    its own tokens give them: logits of other products and other attention kernels,
    about two dozen binary16 roundings of 2^-11 apart behind norms that may stretch them
    a few times, are within 2e-2 of the largest logit; a log probability, the difference
    of a logit and a mean of logits, within twice that."""
    n, beams = 12, 3
    (prompt,) = prompts(40)
    tokens, scores, _ = example.search(example.Decoder(pages=256, seed=3), [prompt], beams, n, end=7)
    for b in range(beams):
        model, total, bound = example.Decoder(seed=3), 0.0, 0.0
        model.step(prompt[:-1])
        model.keep(list(range(len(prompt) - 1)))
        text = prompt[-1:] + tokens[0, b].tolist()
        for now, following in zip(text, text[1:]):
            logits = model.step([now])[0].double()
            model.keep([0])
            total += float(torch.log_softmax(logits, 0)[following])
            bound += 2 * 2e-2 * float(logits.abs().max())
        assert abs(total - float(scores[0, b])) <= bound


def test_the_program_runs(example, monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["beam_search.py", "--tokens", "10", "--beams", "3"])
    example.main()
    assert "the same tokens and scores" in capsys.readouterr().out
