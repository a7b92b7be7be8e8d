"""Rounds of drafted tokens as a program runs them: tree, append, attention, sampling, acceptance and compaction, eager and captured."""
import os
import sys

import numpy as np
import pytest
import torch

import _draft_ref as plain

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def state(dec):
    return [x.clone() for cache in dec.caches for x in cache] + [dec.lens.clone(), dec.last.clone()]


def reset(dec, to):
    for x, y in zip([x for cache in dec.caches for x in cache] + [dec.lens, dec.last], to):
        x.copy_(y)


@pytest.mark.parametrize("prompt,rounds,seqs,temperature", [(60, 4, 1, 0.0), (90, 5, 3, 0.7)])
def test_the_example_runs(prompt, rounds, seqs, temperature):
    import drafted_decoding
    tokens, distance = drafted_decoding.run(prompt, rounds, seqs, temperature)
    assert 1 <= tokens <= 4 + 1
    # Every code in either cache is a few roundings of half a step, 2^-4, from its value at most (a page's exponent grows by a few steps at
    # most, as its values do; small ones round to a fixed step, which is less than that of the largest's 2^-4); the layer below adds the like again.
    assert distance < 0.25


@pytest.mark.parametrize("seqs,temperature", [(1, 0.0), (4, 0.0), (3, 0.8)])
def test_each_step_of_a_round_is_its_definition(seqs, temperature):
    import drafted_decoding as ex
    import paper_2605_20315_amd as mq
    dec, texts, draws = ex.start(70, 6, seqs, temperature, 3)
    cu, host = dec.cu_q.cpu().numpy(), lambda t: t.cpu().numpy()
    for u in draws:
        dec.uniform.copy_(u)
        tokens, kv_lens, last = dec.draft(), dec.lens + dec.nodes, dec.last.clone()
        tree, positions = mq.mq_draft_tree(dec.parents, dec.cu_q, kv_lens, dec.words)
        masks, depth = plain.tree(ex.PARENTS * seqs, cu, host(kv_lens), dec.words)
        assert np.array_equal(host(tree), masks) and np.array_equal(host(positions), depth)
        logits = dec.forward(tokens, dec.cu_q, kv_lens, dec.caches, tree, positions)
        sampled = mq.mq_sample(logits, dec.uniform, dec.temperature)
        rows = logits.float().cpu().numpy()
        assert host(sampled).tolist() == [plain.sample(x, d, np.float32(temperature)) for x, d in zip(rows, host(u))]
        path, counts, ends, lens = mq.mq_draft_accept(dec.parents, tokens, sampled, dec.cu_q, kv_lens)
        want = plain.accept(np.array(ex.PARENTS * seqs), host(tokens), host(sampled), cu, host(kv_lens))
        for got, w in zip((path, counts, ends, lens), want):
            assert np.array_equal(host(got), w)
        for cache in dec.caches:
            want = [host(x).copy() for x in cache]
            mq.kv8_compact(*cache, dec.page_table, dec.cu_q, kv_lens, path, counts)
            plain.compact(*want, host(dec.page_table), cu, host(kv_lens), host(path), host(counts))
            for got, w in zip(cache, want):
                assert np.array_equal(host(got), w)
        # what is kept begins with the token that the round before ended in
        new = dec.kept(tokens, path, counts, ends)
        assert [n[0] for n in new] == last.tolist() and lens.tolist() == [len(t) + len(n) for t, n in zip(texts, new)]
        for text, n in zip(texts, new):
            text += n
        dec.lens.copy_(lens)
        dec.last.copy_(ends)


def test_without_chance_the_text_is_that_of_single_steps():
    """The head's margins are far above what roundings move (a logit of sqrt(512) against chance ones of about 1, and about 0.1 from attention)."""
    import drafted_decoding as ex
    dec, texts, draws = ex.start(50, 8, 2, 0.0, 5)
    first = dec.last.tolist()
    made = [[], []]
    for _ in draws:
        for m, new in zip(made, dec.kept(*dec.round())):
            m += new
    for m, token in zip(made, first):
        assert len(m) >= len(draws)
        for got in m:
            assert got == token
            token = int(dec.after[token])
    assert sum(len(m) for m in made) > 2 * 2 * len(draws)  # the drafter is right often enough that paths are long


def test_rounds_replayed_from_a_graph_are_those_run_eagerly():
    """Two graphs on one workspace, with eager rounds, copies and synchronisations between the replays."""
    import drafted_decoding as ex
    dec, texts, draws = ex.start(300, 7, 3, 0.8, 11)
    begin, eager = state(dec), []
    for u in draws:
        dec.uniform.copy_(u)
        out = dec.round()
        eager.append([x.clone() for x in out] + state(dec))
    reset(dec, begin)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = dec.round()
        graphs.append((graph, out))
    reset(dec, begin)
    side = torch.cuda.Stream()
    for i, (u, want) in enumerate(zip(draws, eager)):
        dec.uniform.copy_(u)
        if i % 3 == 2:
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                out = dec.round()
            torch.cuda.current_stream().wait_stream(side)
            torch.cuda.synchronize()
        else:
            graph, out = graphs[i % 2]
            graph.replay()
        for got, w in zip(list(out) + state(dec), want):
            assert torch.equal(got, w), i
