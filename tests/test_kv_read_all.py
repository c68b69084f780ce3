"""Reads that make their own results: no row of them is what the memory held before."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import kv
    return kv


def ints(v):
    return torch.tensor(np.asarray(v, np.int32).reshape(np.shape(v)), device="cuda")


def litter(*sizes):
    """Memory of these tensors' sizes, given back with NaN in every element of 16 bits."""
    kept = [torch.full(s, -1, dtype=torch.int16, device="cuda") for s in sizes for _ in range(2)]
    del kept


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("lens,total", [([], 5), ([0], 3), ([3], 3), ([3], 4), ([1, 0, 40, 7], 1000), ([20] * 300, 7001),
                                        ([0, 0], 1)])
def test_rows_past_the_last_sequence(K, bits, dtype, lens, total):
    """Rows that no sequence has are zeros; the others are what they are in a result that the caller gives, whose other rows stay."""
    H, D, page = 2, 48, 8
    n = len(lens)
    c = K.PagedCache.new(2, sum(-(-x // page) for x in lens) + 1, page, H, D, max(1, n), 6, dtype, bits=bits)
    slot, q = ints(np.arange(n)), ints(np.concatenate([[0], np.cumsum(lens)]))
    used = sum(lens)
    x = [torch.randn((used, H, D), generator=torch.Generator("cuda").manual_seed(s), device="cuda", dtype=dtype)
         for s in (1, 2)]
    assert c.extend(slot, ints(lens)).tolist() == [1] * n
    c.append(1, *x, slot, q)
    own = tuple(torch.full((total, H, D), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    c.read(1, slot, q, out=own)
    for _ in range(3):
        litter((total, H, D))
        for got, mine in zip(c.read(1, slot, q, total=total), own):
            assert torch.equal(got[:used].view(torch.int16), mine[:used].view(torch.int16))
            assert bool((got[used:].view(torch.int16) == 0).all())
            assert bool((mine[used:] == 7.0).all())


def test_another_stream_and_a_graph(K):
    """Zeros in a read on a stream that is given, and in replays of a captured one, whose memory others wrote in between."""
    c = K.PagedCache.new(1, 8, 8, 2, 64, 2, 4, bits=8)
    slot, q = ints([1]), ints([0, 9])
    c.extend(slot, ints([9]))
    x = torch.randn((9, 2, 64), device="cuda").bfloat16()
    c.append(0, x, x, slot, q)
    want = torch.zeros((50, 2, 64), dtype=torch.bfloat16, device="cuda")
    c.read(0, slot, q, out=(want, want.clone()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        litter((50, 2, 64))
    got = c.read(0, slot, q, total=50, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(t, want) for t in got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = c.read(0, slot, q, total=50)
    for _ in range(4):
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, want) for t in got)
