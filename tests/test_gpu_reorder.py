"""Reordering of beams' cached tokens: exact, every layer, nothing else touched."""
import pytest
import torch

from paper_2609_26100_amd import ops

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def bits(x):
    return x.view(torch.int16 if x.dtype == torch.float16 else torch.int32)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Beams:
    def __init__(self, groups, beams, shared, lengths, layers=2, heads=2, hd=64, t=torch.float16, seed=0, spare=1):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.groups, self.beams, self.shared, self.lengths = groups, beams, shared, lengths
        n = groups * beams
        own = max(-(-x // 16) for x in lengths) + spare
        width = max(shared) + own
        ids = torch.randperm(groups * max(shared) + n * own + 3, generator=g, device=DEV).to(torch.int32)
        total = ids.numel()
        self.table = torch.empty(n, width, dtype=torch.int32, device=DEV)
        at = 0
        for i in range(groups):
            k = shared[i]
            self.table[i * beams:(i + 1) * beams, :k] = ids[at:at + k]
            at += k
        for s in range(n):
            k = width - shared[s // beams]
            k = min(k, own)
            self.table[s, shared[s // beams]:shared[s // beams] + k] = ids[at:at + k]
            self.table[s, shared[s // beams] + k:] = -1
            at += k
        b = torch.int16 if t == torch.float16 else torch.int32
        info = torch.iinfo(b)
        self.pages = torch.randint(info.min, info.max, (layers, total, 2, heads, 16 * hd), generator=g, device=DEV,
                                   dtype=b).view(t)

    def want(self, parents, max_own=None):
        out, table = bits(self.pages).clone(), self.table.cpu()
        old = out.clone()
        for g in range(self.groups):
            for b in range(self.beams):
                p = parents[g][b]
                if not 0 <= p < self.beams or p == b:
                    continue
                s, d = g * self.beams + p, g * self.beams + b
                for i in range(-(-max(self.lengths[s], 0) // 16)):
                    pg = self.shared[g] + i
                    if (max_own is not None and i >= -(-max_own // 16)) or pg >= table.shape[1]:
                        break
                    if 0 <= table[s, pg] < out.shape[1] and 0 <= table[d, pg] < out.shape[1]:
                        out[:, table[d, pg]] = old[:, table[s, pg]]
        return out

    def lens(self):
        return ints([n + 16 * self.shared[i // self.beams] if n > 0 else n for i, n in enumerate(self.lengths)])

    def check(self, parents, **kw):
        want = self.want(parents, kw.get("max_own"))
        shared = None if not any(self.shared) else ints(self.shared)
        ops.reorder_pages(self.pages, self.table, ints(parents), self.lens(), shared, **kw)
        assert torch.equal(bits(self.pages), want)


@pytest.mark.parametrize("t", [torch.float16, torch.float32])
@pytest.mark.parametrize("layers,heads,hd", [(1, 1, 64), (3, 5, 128)])
def test_maps(t, layers, heads, hd):
    for parents in ([0, 1, 2, 3], [1, 0, 3, 2], [1, 2, 3, 0], [2, 2, 2, 2], [0, 0, 1, 1], [3, 1, 1, 0]):
        Beams(1, 4, [2], [40, 33, 16, 1], layers, heads, hd, t, seed=len(parents)).check([parents])


@pytest.mark.parametrize("beams", [1, 2, 3, 5, 8, 9, 16, 17, 32])
def test_numbers_of_beams(beams):
    g = torch.Generator().manual_seed(beams)
    groups = 3
    lengths = torch.randint(0, 70, (groups * beams,), generator=g).tolist()
    parents = torch.randint(0, beams, (groups, beams), generator=g).tolist()
    Beams(groups, beams, [0, 3, 1], lengths, seed=beams).check(parents)
    rot = [[(b + 1) % beams for b in range(beams)]] * groups
    Beams(groups, beams, [0, 0, 0], lengths, seed=beams).check(rot)


def test_bounds_and_what_is_left():
    b = Beams(2, 3, [1, 4], [50, 20, 0, 33, 1, 17], seed=1)
    b.check([[1, 0, 0], [5, -1, 0]])                 # parents outside the group's beams stay
    for most in (0, 1, 16, 17, 1000):
        Beams(2, 3, [1, 4], [50, 20, 0, 33, 1, 17], seed=2).check([[1, 2, 0], [1, 2, 0]], max_own=most)
    b = Beams(1, 3, [1], [50, 20, 33], seed=3, spare=0)
    b.table[0, 2], b.table[1, 1], b.table[2, 3] = -1, b.pages.shape[1], 2 ** 31 - 1
    b.check([[2, 0, 1]])
    b = Beams(1, 2, [0], [-5, 16 * 1000], seed=4)    # lengths outside the page table
    b.check([[1, 0]])


def test_captured_and_replayed():
    b = Beams(2, 4, [1, 0], [40, 33, 16, 1, 5, 30, 31, 32], seed=5)
    parents, lens, shared = ints([[0] * 4] * 2), b.lens(), ints(b.shared)
    ops.reorder_pages(b.pages, b.table, parents, lens, shared, max_own=40)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.reorder_pages(b.pages, b.table, parents, lens, shared, max_own=40)
    for p in ([[1, 0, 3, 2], [3, 3, 0, 0]], [[2, 0, 1, 1], [0, 1, 2, 3]], [[1, 2, 3, 0], [1, 2, 3, 0]]):
        want = b.want(p)
        parents.copy_(torch.tensor(p, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(bits(b.pages), want)


def test_beyond_four_gib():
    b = Beams(1, 2, [0], [64, 64], layers=1, heads=8, hd=128, seed=6, spare=0)
    big = torch.zeros(2, 40000, 2, 8, 16 * 128, dtype=torch.float16, device=DEV)   # 2.6 GB a layer
    where = ints([[39990 + i for i in range(4)], [39000 + i for i in range(4)]])
    for s in range(2):
        big[:, where[s].long()] = b.pages[0, b.table[s].long()]
    a, c = big[:, where[0].long()].clone(), big[:, where[1].long()].clone()
    ops.reorder_pages(big, where, ints([[1, 0]]), ints([64, 64]))
    assert torch.equal(bits(big[:, where[0].long()]), bits(c)) and torch.equal(bits(big[:, where[1].long()]), bits(a))


def test_on_a_stream_of_its_own():
    b = Beams(1, 4, [2], [40, 33, 16, 1], seed=7)
    want = b.want([[3, 2, 1, 0]])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ops.reorder_pages(b.pages, b.table, ints([[3, 2, 1, 0]]), b.lens(), ints(b.shared))
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(bits(b.pages), want)


def test_refusals():
    b = Beams(1, 4, [2], [40, 33, 16, 1])
    lens, shared, par = b.lens(), ints(b.shared), ints([[0, 1, 2, 3]])
    for bad in (dict(parents=par[0]), dict(parents=par[:, :3]), dict(parents=par.long()), dict(lengths=lens[:3]),
                dict(shared=ints([1, 2])), dict(pages=b.pages.bfloat16()), dict(page_table=b.table[0])):
        with pytest.raises(ValueError):
            ops.reorder_pages(**dict(dict(pages=b.pages, page_table=b.table, parents=par, lengths=lens, shared=shared),
                                     **bad))
    with pytest.raises(ops.abi.TSSError):
        ops.reorder_pages(b.pages, b.table, par, lens, shared, max_own=-1)
