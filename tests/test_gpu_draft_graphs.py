"""Sampling and attention of drafted tokens captured into graphs: replayed several times, with other inputs in the same memory, eager work of the
program between the replays, and a workspace that two graphs share."""
import numpy as np
import pytest
import torch

import paper_2605_20315_amd as mq
from test_gpu_kv8_attention import dev
from test_gpu_kv8_tree_attention import Problem

pytestmark = pytest.mark.gpu


def captured(call):
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    return graph, out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_sampling(dtype):
    gen = torch.Generator("cuda").manual_seed(3)
    sizes = [(40, 20001), (3, 150001), (60, 700)]
    ws = torch.empty(max(mq.mq_sample_workspace_bytes(*s) for s in sizes), dtype=torch.uint8, device="cuda")
    calls, fills = [], []
    for rows, V in sizes:
        x, u = torch.empty(rows, V, dtype=dtype, device="cuda"), torch.empty(rows, device="cuda")
        have = {"temperature": torch.empty(rows, device="cuda"), "top_k": torch.empty(rows, dtype=torch.int32, device="cuda"),
                "top_p": torch.empty(rows, device="cuda"), "min_p": torch.empty(rows, device="cuda")}

        def fill(x=x, u=u, have=have):
            x.copy_(3 * torch.randn(x.shape, device="cuda", generator=gen))
            u.copy_(torch.rand(u.shape, device="cuda", generator=gen))
            have["temperature"].copy_(1.5 * torch.rand(u.shape, device="cuda", generator=gen) - 0.1)
            have["top_k"].copy_(torch.randint(0, 400, u.shape, device="cuda", generator=gen))
            have["top_p"].copy_(0.5 + 0.6 * torch.rand(u.shape, device="cuda", generator=gen))
            have["min_p"].copy_((0.2 * torch.rand(u.shape, device="cuda", generator=gen) - 0.1).clamp_min(0))
        fill()
        fills.append(fill)
        calls += [lambda x=x, u=u, have=have: mq.mq_sample(x, u, **have, workspace=ws), lambda x=x, u=u, have=have: mq.mq_sample(x, u, have["temperature"], workspace=ws)]
    graphs = [captured(call) for call in calls]
    for _ in range(4):
        for fill in fills:
            fill()
        for call, (graph, out) in zip(calls, graphs):
            want = call()
            out.fill_(-7)
            graph.replay()
            assert torch.equal(out, want)
            ws.fill_(0xFF)
        torch.cuda.synchronize()


def test_attention_of_other_lengths_and_trees():
    r = np.random.default_rng(5)
    problems = [Problem(5, [20, 60, 9], [9000, 300, 4000], 8, 2, 128, 64), Problem(6, [4] * 40, [900] * 40, 8, 8, 64, 16)]
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    calls, states = [], []
    for p in problems:
        args, positions = p.device(), dev(p.positions)
        states.append((p, args[7], args[8], positions))
        calls.append(lambda p=p, args=args, positions=positions: mq.kv8_tree_attention(*args, p.scale, 700, positions, workspace=ws))
    graphs = [captured(call) for call in calls]
    for turn in range(5):
        for p, lens, tree, positions in states:
            n = np.diff(p.cu)
            new = np.array([r.integers(m, total + 1) for m, total in zip(n, p.lens)], np.int32) if turn else p.lens
            lens.copy_(dev(new))
            tree.copy_(dev(r.integers(-(2 ** 31), 2 ** 31, p.tree.shape).astype(np.int32)))
            positions.copy_(dev(r.integers(0, int(p.lens.max()), p.positions.shape).astype(np.int32)))
        for call, (graph, out) in zip(calls, graphs):
            want = call()
            out.fill_(float("nan"))
            graph.replay()
            assert torch.equal(out.view(torch.int16), want.view(torch.int16))
            ws.fill_(0xFF)
        torch.cuda.synchronize()


def test_two_streams_sample_at_once():
    gen = torch.Generator("cuda").manual_seed(9)
    xs = [3 * torch.randn(70, 40001, device="cuda", generator=gen) for _ in range(2)]
    u, p = torch.rand(70, device="cuda", generator=gen), torch.full((70,), 0.9, device="cuda")
    want = [mq.mq_sample(x, u, top_p=p) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for stream, x, out in zip(streams, xs, got):
            with torch.cuda.stream(stream):
                out.append(mq.mq_sample(x, u, top_p=p))
    torch.cuda.synchronize()
    assert all(torch.equal(y, w) for out, w in zip(got, want) for y in out)
