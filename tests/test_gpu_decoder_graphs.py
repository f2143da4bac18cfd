"""Captured calls of the decoder operators, replayed after eager calls of the same objects that need more workspace than the captured ones had."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def taken(lo, size):
    """Tensors of a pattern, as many as would fill what the allocator has been given back of [lo, lo + size); none of them may lie there."""
    made = [torch.full((size,), 0xA5, dtype=torch.uint8, device="cuda") for _ in range(64)]
    assert not any(t.data_ptr() < lo + size and lo < t.data_ptr() + size for t in made), "the captured call's workspace was given back"
    return made


def replayed(graph, op, call, larger, change, held):
    """`held` objects' graph of `call` after `larger`: its workspace is still its own, and every replay is the eager call's result."""
    lo, size = op.workspace.data_ptr(), op.workspace.numel()
    larger()
    torch.cuda.synchronize()
    assert op.workspace.numel() > size
    made = taken(lo, size)
    for i in range(4):
        change(i)
        want = call().clone()
        held.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, want)
        assert all((t == 0xA5).all() for t in made)


@pytest.mark.parametrize("warm", [True, False])
def test_products(warm):
    """Rows quantised by a launch of their own (17 blocks of inputs: too many codes for the kernel that quantises them itself)."""
    from paper_2007_12216_amd.decoder import Fp8Linear
    g = torch.Generator().manual_seed(0)
    make = lambda *shape: torch.randn(*shape, generator=g).to(torch.bfloat16).cuda()
    layer, x, many = Fp8Linear.from_weights(make(300, 2100)), make(64, 2100), make(2000, 2100)
    y, x0 = torch.empty(64, 300, dtype=torch.bfloat16, device="cuda"), x.clone()
    if warm:
        layer.forward(x, y)
    else:
        Fp8Linear.from_weights(make(300, 2100)).forward(x, y)  # (the kernels' first launch)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(x, y)
    replayed(graph, layer, lambda: layer.forward(x), lambda: layer.forward(many), lambda i: x.copy_(x0 * (1 + i)), y)


@pytest.mark.parametrize("warm", [True, False])
def test_attention(warm):
    """One long request whose positions several workgroups share, then eight of them."""
    from paper_2007_12216_amd.decoder import Cache4, CacheAttention
    rng = np.random.default_rng(1)
    to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    pages, page, kv, dim = 130, 16, 2, 128
    tensors = [to(rng.integers(0, 256, (pages, kv, page, dim // 2), dtype=np.uint8)) if i % 2 == 0 else to(rng.integers(124, 129, (pages, kv, page, dim // 32), dtype=np.uint8)) for i in range(4)]
    cache = Cache4(pages, page, kv, dim, tensors=tensors)
    table, lens = to(rng.permutation(pages)[None].astype(np.int32)), to(np.array([2000], dtype=np.int32))
    q0 = torch.randn(8, 8, dim, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    q, out, rows = q0[:1].clone(), torch.empty(1, 8, dim, dtype=torch.bfloat16, device="cuda"), to(np.arange(9, dtype=np.int32))
    op = CacheAttention(cache, 8)
    (op if warm else CacheAttention(cache, 8)).forward(q, table, lens, rows[:2], max_fresh=1, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.forward(q, table, lens, rows[:2], max_fresh=1, out=out)
    larger = lambda: op.forward(q0, table.repeat(8, 1), lens.repeat(8), rows, max_fresh=1)
    replayed(graph, op, lambda: op.forward(q, table, lens, rows[:2], max_fresh=1), larger, lambda i: q.copy_(q0[i:i + 1]), out)


def test_every_capture_keeps_its_own():
    """Three captures, each after a call that needed more than the one before; eager calls alone keep nothing but the last workspace."""
    from paper_2007_12216_amd.decoder import Fp8Linear
    g = torch.Generator().manual_seed(2)
    make = lambda *shape: torch.randn(*shape, generator=g).to(torch.bfloat16).cuda()
    layer = Fp8Linear.from_weights(make(300, 2100))
    sizes, xs, ys, graphs = (40, 90, 400), [], [], []
    for n in sizes:
        xs.append(make(n, 2100))
        ys.append(layer.forward(xs[-1]).clone())
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            layer.forward(xs[-1], ys[-1])
    layer.forward(make(1000, 2100))
    made = [torch.full((1 << 20,), 0xA5, dtype=torch.uint8, device="cuda") for _ in range(16)]
    wanted = [layer.forward(x).clone() for x in xs]
    for _ in range(3):
        for graph, y, want in zip(graphs, ys, wanted):
            y.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want)
    assert all((t == 0xA5).all() for t in made)
    before = torch.cuda.memory_allocated()
    for n in (1100, 1200, 1300, 1400):
        layer.forward(make(n, 2100))
    assert torch.cuda.memory_allocated() - before < 2 * 1400 * 2176
