"""paged_copy_pages: exact copies, and nothing else touched."""

import pytest
import torch

pytestmark = pytest.mark.gpu


def _P():
    import paper_2609_36899_amd as P
    return P


def _ids(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


SHAPES = [(16, 576, torch.bfloat16), (16, 640, torch.uint8), (16, torch.float32), (3, torch.uint8),
          (1, torch.float32), (8, 16, 128, torch.bfloat16), (7, 11, torch.int16), (70001, torch.uint8)]


def _pool(pages, shape):
    *dims, dtype = shape
    return torch.randint(0, 100, (pages, *dims), device="cuda").to(dtype)


@pytest.mark.parametrize("shape", SHAPES)
def test_one_pool(shape):
    pool = _pool(20, shape)
    want = pool.clone()
    src, dst = _ids(3, 3, 7, 19, 0), _ids(1, 18, 4, 2, 9)
    want[dst.long()] = want[src.long()]
    _P().paged_copy_pages(pool, src, dst)
    assert torch.equal(pool, want)


@pytest.mark.parametrize("n", [1, 8, 17, 40])
def test_many_pools_together(n):
    pools = [_pool(30, SHAPES[i % len(SHAPES)]) for i in range(n)]
    want = [p.clone() for p in pools]
    order = torch.randperm(30, device="cuda")
    src, dst = order[:12].int(), order[12:24].int()
    for p in want:
        p[dst.long()] = p[src.long()]
    _P().paged_copy_pages(pools, src, dst)
    assert all(torch.equal(p, w) for p, w in zip(pools, want))


def test_unaligned_pools():
    flat = torch.randint(0, 256, (10 * 48 + 5,), device="cuda").to(torch.uint8)
    for off in (1, 4, 0):
        pool = flat[off:off + 480].view(10, 48)
        want = flat.clone()
        want[off:off + 480].view(10, 48)[9] = pool[2]
        _P().paged_copy_pages(pool, _ids(2), _ids(9))
        assert torch.equal(flat, want)


def test_ids_outside_the_pool_copy_nothing():
    pool = _pool(6, SHAPES[0])
    want = pool.clone()
    want[1] = want[0]
    _P().paged_copy_pages(pool, _ids(-1, 2, 6, 3, 4, 0, 1 << 30), _ids(2, -5, 3, 6, 4, 1, 5))
    assert torch.equal(pool, want)


def test_no_pairs_and_offsets_past_32_bits():
    n = (1 << 32) // (16 * 640) + 30
    pool = torch.zeros(n, 16, 640, dtype=torch.uint8, device="cuda")
    pool[n - 1], pool[2] = 77, 55
    _P().paged_copy_pages(pool, _ids(), _ids())
    _P().paged_copy_pages(pool, _ids(n - 1, 2), _ids(5, n - 3))
    assert (pool[5] == 77).all() and (pool[n - 3] == 55).all()
    assert int(torch.count_nonzero(pool.view(n, -1).any(1))) == 4


def test_captured_copies_follow_the_pairs():
    pool = _pool(12, SHAPES[1])
    src, dst = _ids(0, 1), _ids(6, 7)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        _P().paged_copy_pages([pool], src, dst)
    for a, b in [((0, 1), (6, 7)), ((2, 2), (8, 9)), ((5, -1), (10, 11))]:
        want = pool.clone()
        for s, d in zip(a, b):
            if s >= 0:
                want[d] = want[s]
        src.copy_(_ids(*a))
        dst.copy_(_ids(*b))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(pool, want)
