"""Appends to and reads of caches by more tokens than one pass of the largest grid has: 65,536 workgroups of eight."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import codes_ref  # noqa: E402

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ONE_PASS = 8 * 65536
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def ints(v):
    return torch.tensor(np.asarray(v, np.int32).reshape(np.shape(v)), device="cuda")


@pytest.mark.parametrize("kind,bits,heads", [("bf16", 8, 1), ("f16", 8, 2), ("bf16", 16, 1)])
def test_second_pass(kind, bits, heads):
    """Sequences that begin, end and have holes on both sides of the first pass's last token, with a partial last workgroup."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import kv
    D, page = 16, 64
    lens = [ONE_PASS - 3, 2, 0, 90_003, 1, 70]
    n = sum(lens)
    assert ONE_PASS < n < 2 * ONE_PASS and n % 8
    c = kv.PagedCache.new(1, sum(-(-x // page) for x in lens), page, heads, D, len(lens), -(-max(lens) // page), TYPES[kind],
                          bits=bits)
    slot, q = ints(np.arange(len(lens))), ints(np.concatenate([[0], np.cumsum(lens)]))
    assert c.extend(slot, ints(lens)).tolist() == [1] * len(lens)
    g = torch.Generator("cuda").manual_seed(bits)
    k, v = (torch.randn((n, heads, D), generator=g, device="cuda").to(TYPES[kind]) for _ in range(2))
    c.append(0, k, v, slot, q)
    lost = slice(ONE_PASS - 3 + 2 + page, ONE_PASS - 3 + 2 + 3 * page)  # two pages of the fourth sequence
    c.release(ints([3]), ints([page]), ints([3 * page]))
    for got, x in zip(c.read(0, slot, q, total=n), (k, v)):
        want = codes_ref.quantise(x.double().cpu().numpy(), kind)[2] if bits == 8 else x.double().cpu().numpy()
        want[lost] = 0
        assert np.array_equal(got.double().cpu().numpy(), want)
