"""The calls of examples/attention_step.py together: gradients of the whole chain against differences, both types, a captured step."""
import importlib.util
import os

import pytest
import torch

import blockgen as bg
from paper_2409_14939_amd import binding as B

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("attention_step", os.path.join(ROOT, "examples", "attention_step.py"))
ex = importlib.util.module_from_spec(spec)
spec.loader.exec_module(ex)
WIDTH, HEADS, KV, HEAD, RELATIONS, CLASSES = 40, 6, 2, 11, 4, 13


def setting(dtype):
    blk = bg.make_config(1).blocks[0]
    ip, ix = torch.from_numpy(blk.indptr).cuda(), torch.from_numpy(blk.indices).cuda()
    g = torch.Generator().manual_seed(1)
    X = torch.randn(blk.num_src, WIDTH, generator=g).to(dtype).cuda()
    relation = torch.randint(-1, RELATIONS, (blk.num_edges,), generator=g, dtype=torch.int32).cuda()
    labels = torch.randint(-1, CLASSES, (blk.num_dst,), generator=g).cuda()
    dloss = (0.5 + torch.rand(blk.num_dst, generator=g)).cuda()
    p = ex.make_params(WIDTH, HEADS, KV, HEAD, RELATIONS, CLASSES, dtype)
    p["bias"] = torch.randn(RELATIONS, HEADS, generator=g).cuda()
    block = (ip, ix, B.fastgl_block_plan_create(ip, ix, blk.num_src, B.PLAN_ALL | B.PLAN_PERM))
    return p, block, relation, X, labels, dloss


def step(p, block, relation, X, labels, dloss):
    loss, kept = ex.forward(p, block, relation, X, labels, HEADS, KV)
    grads, dX = ex.backward(p, block, relation, X, labels, kept, dloss, HEADS, KV)
    return loss, grads, dX


def test_gradients_of_the_chain_against_differences():
    p, block, relation, X, labels, dloss = setting(torch.float32)
    _, grads, dX = step(p, block, relation, X, labels, dloss)

    def value(p, X):
        return (ex.forward(p, block, relation, X, labels, HEADS, KV)[0].double() * dloss.double()).sum().item()
    gen = torch.Generator().manual_seed(5)
    for name in [*grads, "X"]:
        v, g = (X, dX) if name == "X" else (p[name], grads[name])
        # along the gradient itself and a random direction: the change is far above the losses' float32 noise
        way = g.double() / g.double().norm() + 0.5 * torch.randn(v.shape, generator=gen, dtype=torch.float64).cuda() / v.numel() ** 0.5
        size = 1e-3 * max(v.double().norm().item(), 1.0) / way.norm().item()
        up, down = (v.double() + size * way).float(), (v.double() - size * way).float()
        along = ((up.double() - down.double()) * g.double()).sum().item()
        if name == "X":
            change = value(p, up) - value(p, down)
        else:
            change = value({**p, name: up}, X) - value({**p, name: down}, X)
        # third-order term of a central difference over a thousandth of the parameter's size, and float32 noise of 200 losses
        assert abs(change - along) <= 1e-2 * abs(along) + 1e-3, (name, change, along)


def test_both_types_agree():
    out = []
    for dtype in (torch.float32, torch.bfloat16):
        p, block, relation, X, labels, dloss = setting(dtype)
        loss, grads, dX = step(p, block, relation, X, labels, dloss)
        out.append([loss, dX, *grads.values()])
    for a, b in zip(*out):
        # inputs, weights and some ten results on the way are rounded to 8 bits (2^-8 each, independent)
        assert ((a.double() - b.double()).norm() / a.double().norm()).item() < 12 * 2.0 ** -8


def test_a_captured_step():
    """The whole step in one graph, replayed on other inputs with eager steps between."""
    p, block, relation, X, labels, dloss = setting(torch.bfloat16)
    inputs = [X, (X.float() * 0.5 + 1.0).to(X.dtype)]
    eager = []
    for x in inputs:
        loss, grads, dX = step(p, block, relation, x, labels, dloss)
        eager.append([loss.clone(), dX.clone(), *(g.clone() for g in grads.values())])
    held = X.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step(p, block, relation, held, labels, dloss)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            loss, grads, dX = step(p, block, relation, held, labels, dloss)
    torch.cuda.current_stream().wait_stream(side)
    for n in (0, 1, 1, 0):
        held.copy_(inputs[n])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip([loss, dX, *grads.values()], eager[n]):
            assert torch.equal(a, b)
        step(p, block, relation, inputs[1 - n], labels, dloss)


def test_the_example_runs():
    ex.main()
