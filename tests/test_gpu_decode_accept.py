"""GPU tests of pipeline.Decode.accept: a sequence whose count or path is refused is left as it is, its weights too, and what it says
does not reach the others."""
import pytest
import torch

from tests.decode_cases import signed

pytestmark = pytest.mark.gpu
BF, LAYERS, H, G, D, CAP, N = torch.bfloat16, 2, 8, 2, 64, 80, 50


def verified(device, batch, t, budget=0):
    """A Decode whose layers have verified t drafted tokens (a chain) over caches of N tokens."""
    from paper_2604_06746_b200 import pipeline
    dec = pipeline.Decode(LAYERS, H, G, D, CAP, BF, batch=batch, budget=budget, recent=2, max_new=t, decay=0.5, device=device)
    for b in range(batch):                               # (a sequence's numbers do not depend on the batch)
        gen = torch.Generator().manual_seed(b)
        at = slice(b, None, batch)
        for x in (dec.cache.k, dec.cache.v):
            x[at] = torch.randn((LAYERS, G, CAP, D), generator=gen).to(BF).to(device)
        dec.cache.positions[at] = torch.arange(CAP, dtype=torch.int32, device=device)
        dec.cache.weights[at] = torch.rand((LAYERS, G, CAP), generator=gen).to(device)
        dec.cache.lengths[at] = N
    positions = (N + torch.arange(t, dtype=torch.int32, device=device)).repeat(batch, 1)
    for l in range(LAYERS):
        def noise(heads):
            return torch.stack([torch.randn((t, heads, D), generator=torch.Generator().manual_seed(100 * l + b)).to(BF) for b in range(batch)]).to(device)
        q, k, v = noise(H), noise(G), noise(G)
        dec.verify(l, q, k, v, positions, D ** -0.5, torch.empty_like(q))
    torch.cuda.synchronize()
    return dec


def words(counts, path, device):
    return torch.tensor(counts, dtype=torch.int32, device=device), torch.tensor(path, dtype=torch.int32, device=device)


REFUSED = [(6, [0, 1, 2, 3, 4]), (-1, [0, 1, 2, 3, 4]), (2, [1, 1, 0, 0, 0]), (3, [0, 2, 1, 4, 4]), (2, [3, 5, 0, 0, 0]), (1, [-1, 0, 0, 0, 0]),
           (5, [0, 1, 2, 3, 3]), (2, [4, 4, 4, 4, 4])]


@pytest.mark.parametrize("budget", [0, 50])
def test_refused_sequences_stay_as_they_are(cuda_device, budget):
    from paper_2604_06746_b200 import binding
    t, fine = 5, [(3, [0, 2, 4, -7, -7]), (0, [9, 9, 9, 9, 9]), (5, [0, 1, 2, 3, 4])]
    asked = [x for pair in zip(REFUSED[:3], fine) for x in pair] + REFUSED[3:]
    batch = len(asked)
    dec = verified(cuda_device, batch, t, budget)
    before = [x.clone() for x in (dec.cache.k, dec.cache.v, dec.cache.positions, dec.cache.weights)]
    dec.accept(*words([c for c, _ in asked], [p for _, p in asked], cuda_device))
    torch.cuda.synchronize()
    assert dec.ctx.poll_device_status() == binding.ERR_INVALID_ARG
    alone = verified(cuda_device, batch, t, budget)
    alone.accept(*words([c if (c, p) in fine else 0 for c, p in asked], [p if (c, p) in fine else [0] * t for c, p in asked], cuda_device))
    torch.cuda.synchronize()
    assert alone.ctx.poll_device_status() == binding.OK
    after = (dec.cache.k, dec.cache.v, dec.cache.positions, dec.cache.weights)
    other = (alone.cache.k, alone.cache.v, alone.cache.positions, alone.cache.weights)
    for b, (c, p) in enumerate(asked):
        at = slice(b, None, batch)
        if (c, p) in fine:
            n = min(N + c, budget or N + c)
            assert (dec.cache.lengths[at] == n).all()
            assert all(torch.equal(x[at, :, :n], y[at, :, :n]) for x, y in zip(after, other)), b
            assert not torch.equal(after[3][at, :, :N], before[3][at, :, :N])          # (decayed at least)
        else:
            assert (dec.cache.lengths[at] == N).all()
            assert all(torch.equal(x[at], y[at]) for x, y in zip(after, before)), (b, c, p)


def test_wrong_shapes_and_types_change_nothing(cuda_device):
    dec = verified(cuda_device, 2, 3)
    before = dec.cache.weights.clone()
    counts, path = words([1, 1], [[0, 1, 2], [0, 1, 2]], cuda_device)
    for c, p in ((counts.long(), path), (counts, path.long()), (counts[:1], path), (counts, path[:1]), (counts, path[:, :2]), (counts.cpu(), path),
                 (counts, path.cpu())):
        with pytest.raises(ValueError):
            dec.accept(c, p)
        torch.cuda.synchronize()
        assert torch.equal(dec.cache.weights, before) and (dec.cache.lengths == N).all()
    dec.accept(counts, path)                               # the drafts are still there
    assert (dec.cache.lengths == N + 1).all()


def test_captured_acceptance_follows_the_words(cuda_device):
    """verify and accept in one graph, replayed with other counts and paths, refused ones among them."""
    from paper_2604_06746_b200 import binding, pipeline
    t, batch = 4, 2
    dec = pipeline.Decode(LAYERS, H, G, D, CAP, BF, batch=batch, budget=20, recent=2, max_new=t, device=cuda_device)
    counts, path = words([0, 0], [[0] * t] * 2, cuda_device)
    gen = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((batch, t, x, D), generator=gen).to(BF).to(cuda_device) for x in (H, G, G))
    positions, out = torch.zeros((batch, t), dtype=torch.int32, device=cuda_device), torch.empty_like(q)
    tree = torch.tensor([[signed((2 << i) - 1) for i in range(t)]] * batch, dtype=torch.int64, device=cuda_device)

    def go():
        for l in range(LAYERS):
            dec.verify(l, q, k, v, positions, 0.125, out, tree)
        dec.accept(counts, path)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        go()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            go()
        want = [0, 0]
        for c, p in (([2, 1], [[0, 1, 9, 9], [3, 0, 0, 0]]), ([4, 5], [[0, 1, 2, 3]] * 2), ([1, 1], [[4, 0, 0, 0], [0, 0, 0, 0]])):
            counts.copy_(torch.tensor(c, dtype=torch.int32))
            path.copy_(torch.tensor(p, dtype=torch.int32))
            graph.replay()
            for b in range(batch):
                ok = 0 <= c[b] <= t and all(0 <= x < t for x in p[b][:c[b]]) and sorted(set(p[b][:c[b]])) == p[b][:c[b]]
                want[b] += c[b] if ok else 0
            side.synchronize()
            assert dec.cache.lengths.view(LAYERS, batch, G).permute(1, 0, 2).reshape(batch, -1).cpu().tolist() == [[w] * (LAYERS * G) for w in want]
    assert dec.ctx.poll_device_status() == binding.ERR_INVALID_ARG
