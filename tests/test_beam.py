"""The beams' selection against the definition in 64 bits: parents and tokens
equal, scores to binary32's rounding."""
import math
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import codes_ref  # noqa: E402

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import beam
    return beam


def check(B, logits, score, beams, picks, done=None, end=0, **kw):
    logits, score = logits.cuda(), torch.as_tensor(score, dtype=torch.float32).cuda()
    d = None if done is None else torch.tensor(done, dtype=torch.int32).cuda()
    got = B.beam_select(logits, score, beams, picks, done=d, end=end, **kw)
    torch.cuda.synchronize()
    with np.errstate(all="ignore"):
        want = codes_ref.select(logits.cpu().double().numpy(), score.cpu().double().numpy(), beams, picks, done, end)
    assert np.array_equal(got[0].cpu().numpy(), want[0])
    assert np.array_equal(got[1].cpu().numpy(), want[1])
    z = got[2].cpu().double().numpy()
    # One rounding to binary32 of score + logit - ln sum.  Of an exponential's factors 2^(n / 256) is right to 2^-52; of e^r
    # the third term, (ln 2 / 512)^3 / 6 < 2^-31.1, is left out, r in steps of ln 2 / 256 is off by 2^-25 and e^r - 1 < 2^-9.5
    # by 2 2^-24 of itself: 2^-33.5 and 2^-32.5, in all 2^-30.  The sum and the largest one that it is divided by are both off
    # by as much: 2^-29, and so is the logarithm.
    fine = np.isfinite(want[2])
    assert np.array_equal(z[~fine], want[2][~fine])
    z, want = np.where(fine, z, 0), (*want[:2], np.where(fine, want[2], 0))
    assert np.all(np.abs(z - want[2]) <= 2.0 ** -24 * np.abs(want[2]) + 2.0 ** -29 + 2.0 ** -40 * np.abs(want[2]))
    return got


def draw(seed, rows, vocab, kind, spread=2.5):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, vocab), generator=g) * spread
    x[torch.arange(rows), torch.randint(0, vocab, (rows,), generator=g)] += 9
    return x.to(TYPES[kind])


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 63, 200, 1024, 1025, 4096, 50001])
@pytest.mark.parametrize("groups,beams,picks", [(1, 1, 1), (3, 4, 8), (2, 5, 5), (1, 32, 64), (5, 8, 16)])
def test_sizes(B, kind, vocab, groups, beams, picks):
    rows = groups * beams
    rng = np.random.default_rng(vocab)
    check(B, draw(vocab + picks, rows, vocab, kind), -rng.random(rows) * 20, beams, picks)


@pytest.mark.parametrize("kind,vocab,groups,beams,picks", [("bf16", 131072, 4, 8, 16), ("f32", 131071, 1, 2, 64),
                                                           ("f16", 400001, 2, 3, 33), ("bf16", 16385, 70, 8, 8),
                                                           ("f32", 8200, 128, 4, 48), ("bf16", 9000, 256, 2, 64)])
def test_large(B, kind, vocab, groups, beams, picks):
    """Several segments a row, of every size that a thread may hold."""
    rows = groups * beams
    check(B, draw(3, rows, vocab, kind), -np.random.default_rng(1).random(rows) * 5, beams, picks)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("beams,picks,vocab", [(32, 64, 300000), (32, 33, 130001), (16, 48, 52767), (5, 64, 90000), (32, 64, 5000)])
@pytest.mark.parametrize("ahead", [0, 1, 2, 8, 31])
def test_leading_beams(B, kind, beams, picks, vocab, ahead):
    """More candidates of a group than are ranked at once, most of the best of them from a few of its beams; few tokens
    allowed; and scores that are alike in all but their last bits."""
    x = draw(ahead, beams, vocab, kind, spread=0.5)
    x[torch.arange(beams), x.float().argmax(1)] = 0
    score = -30 - np.random.default_rng(ahead).random(beams)
    score[np.random.default_rng(ahead + 1).permutation(beams)[:ahead]] += 25
    check(B, x, score, beams, picks)
    y = torch.full_like(x, -math.inf)
    few = torch.arange(ahead, vocab, 997)
    y[:, few] = x[:, few]
    check(B, y, score, beams, picks)
    near = torch.randn((beams, vocab), generator=torch.Generator().manual_seed(vocab)) * 2.0 ** -14 + 1
    check(B, near.to(x.dtype), score, beams, picks)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("skew", [0, 1, 2, 3, 5, 7])
def test_rows_anywhere(B, kind, skew):
    """Rows that begin at any element, any stride apart; what lies between them is not read as theirs."""
    rows, vocab = 6, 1003
    wide = torch.full((rows, vocab + 2 * skew + 1), 1e4).to(TYPES[kind])
    wide[:, skew:skew + vocab] = draw(skew, rows, vocab, kind)
    check(B, wide.cuda()[:, skew:skew + vocab], -np.arange(6.0), 3, 6)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("vocab,picks", [(300, 4), (40000, 16), (40000, 64)])
def test_ties(B, kind, vocab, picks):
    """Equal logits go to the lower token, equal scores to the lower row; plateaus longer than any list."""
    x = torch.zeros((6, vocab))
    x[1::2, ::3] = -0.0
    x[2, 5:] = 1.0
    x[3] = (torch.arange(vocab) % 7).float()
    x[4, -picks // 2:] = 2.0
    x[5] = x[3]
    score = [0.0, 0.0, -1.0, -2.0, -2.0, -2.0]
    check(B, x.to(TYPES[kind]), score, 2, picks)
    check(B, x.to(TYPES[kind]), score, 6, picks)
    check(B, torch.zeros((4, vocab), dtype=TYPES[kind]), [-3.0] * 4, 4, picks)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,vocab,picks", [(2, 9000, 4), (600, 20000, 4), (600, 20000, 40)])
def test_zeros_with_signs(B, kind, rows, vocab, picks):
    """-0 is 0: of both the lower token."""
    x = torch.full((rows, vocab), -1.0)
    x[:, 0:64:8] = -0.0
    x[:, 256:768:8] = 0.0
    x[1::2, 8003:] = -0.0
    check(B, x.to(TYPES[kind]), [-1.0] * rows, 1, picks)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("picks", [1, 16, 32, 33, 64])
def test_plateaus_in_long_rows(B, kind, picks):
    """Few tokens allowed, by -inf or by the type's lowest value; runs of equal logits above and below the last pick's;
    logits in order; pieces of 16 bytes that are full of the same number."""
    rows, vocab = 520, 17000
    g = torch.Generator().manual_seed(picks)
    x = draw(picks, rows, vocab, kind)
    few = torch.rand((rows, vocab), generator=g) < 0.0004
    low = torch.finfo(x.dtype).min
    x[0::8] = torch.where(few[0::8], x[0::8], -math.inf)
    x[1::8] = torch.where(few[1::8], x[1::8], low)
    x[2::8] = (torch.arange(vocab) % 5 == 0).to(x.dtype)
    x[3::8] = (torch.arange(vocab) / 4096).to(x.dtype)
    x[4::8] = (-torch.arange(vocab) / 4096).to(x.dtype)
    x[5::8] = (torch.arange(vocab) // 8 % 64 < picks - 1).to(x.dtype)
    x[6::8] = ((torch.arange(vocab) % 4096 < 8 * (picks - 1)) * 2 + (torch.arange(vocab) % 3 == 0)).to(x.dtype)
    x[7::8] = low
    check(B, x, [-2.0] * rows, 1, picks)
    check(B, x, -torch.rand(rows, generator=g) * 0.1, 8, picks)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("vocab", [50, 5000, 70000])
def test_masks(B, kind, vocab):
    """Forbidden tokens, rows without any left, the type's lowest value as a mask, NaN and infinities."""
    rows = 8
    x = draw(vocab, rows, vocab, kind)
    x[0, 1:] = -math.inf
    x[1] = -math.inf
    x[2, ::2] = torch.finfo(x.dtype).min
    x[3, 3:9] = math.nan
    x[4] = math.nan
    x[5, [7, vocab - 1, 30]] = math.inf
    x[6, 2:] = -math.inf
    x[6, :2] = torch.tensor([math.nan, 1.0])
    x[7] = torch.finfo(x.dtype).min
    for beams, picks in ((8, 16), (1, 4), (2, 50), (4, 8)):
        check(B, x, -np.arange(rows) * 0.5, beams, picks)


@pytest.mark.parametrize("kind,quiet,loud", [("bf16", 0x7fc1, 0x7f81), ("f16", 0x7e01, 0x7c01), ("f32", 0x7fc00001, 0x7f800001)])
@pytest.mark.parametrize("vocab", [40, 9000])
def test_nan_bits(B, kind, quiet, loud, vocab):
    """NaN of either kind and sign, before and after the largest logit of its row, beside infinities and alone."""
    x = draw(6, 6, vocab, kind)
    raw = x.view(torch.int32 if kind == "f32" else torch.int16)
    sign = 0x80000000 if kind == "f32" else 0x8000
    top = 2 ** 32 if kind == "f32" else 2 ** 16
    for r in range(6):
        for i, bits in enumerate((quiet, loud, quiet | sign, loud | sign)):
            at = (torch.arange(0, vocab, 5) + r + i) % vocab
            raw[r, at] = bits - top if bits & sign else bits
    x[4, 2] = math.inf
    x[5] = math.nan
    raw[5, ::2] = loud
    check(B, x, -np.arange(6.0), 3, 6)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_scores(B, kind):
    """Beams that are not there, first steps, scores of any size."""
    x = draw(1, 8, 3000, kind)
    inf, nan = math.inf, math.nan
    for score in ([0, -inf, -inf, -inf, 0, -inf, -inf, -inf], [-inf] * 8, [nan, -1, nan, -inf, -2, nan, nan, nan],
                  [-1e30, -1e30, -3e38, -1, 1e30, 5, 0, -0.0], [inf, 0, inf, 1, -inf, 2, inf, inf]):
        for picks in (3, 8, 20):
            check(B, x, score, 4, picks)


def test_far_logits(B):
    """Logits whose multiples pass 32 bits, large ones among small ones, and none far apart at all."""
    x = draw(2, 6, 5000, "f32")
    x[0] += 2e6
    x[1] *= 1e30
    x[2] -= 5e5
    x[3] = x[3] * 1e-30
    x[4, 17] = 3e38
    x[5] = -3e38
    for beams in (1, 2, 6):
        check(B, x, [-1.0, -2.0, -3.0, -0.5, 0.0, -1.0], beams, 12)


@pytest.mark.parametrize("kind,vocab", [("bf16", 40000), ("f32", 100)])
def test_done(B, kind, vocab):
    """Beams at their end go on by the end token alone, whatever their logits."""
    x = draw(5, 12, vocab, kind)
    x[3] = math.nan
    done = [0, 1, 0, 1, 1, 1, 1, 1, 0, 0, -7, 0]
    score = -np.arange(12.0) * 0.3
    score[6] = -math.inf
    for picks in (2, 4, 10):
        check(B, x, score, 4, picks, done, vocab - 1)
        check(B, x, score, 4, picks, [1] * 12, 0)


def test_sorted_logits(B):
    """Rows in ascending and descending order: the candidates all in one segment, or everywhere."""
    up = torch.linspace(-20, 5, 60000)
    x = torch.stack([up, up.flip(0), up, up.flip(0)])
    for kind in ("f32", "bf16"):
        check(B, x.to(TYPES[kind]), [0.0, -0.1, -5.0, -0.2], 2, 64)
        check(B, x.to(TYPES[kind]), [0.0, -0.1, -5.0, -0.2], 4, 7)


def test_near_scores(B):
    """Candidates of different rows whose scores lie 1e-9 apart keep their order."""
    g = torch.Generator().manual_seed(8)
    base = torch.randn(20000, generator=g) * 2
    x = base.repeat(8, 1)
    for r in range(8):  # a little more weight far below the top moves every score of the row by about 1e-9
        x[r, 19999] = -30.0 + 0.1 * ((r * 5) % 8)
        x[r, 19998] = -9.0
    check(B, x, [-1.0] * 8, 8, 64)


def test_streams_outputs_and_graph(B):
    from paper_2601_21758_amd import ewsjf
    x, score = draw(4, 16, 30000, "bf16").cuda(), -torch.rand(16, generator=torch.Generator().manual_seed(1)).cuda()
    ws = ewsjf.Workspace()
    want = B.beam_select(x, score, 8, 16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = tuple(torch.empty_like(t) for t in want)
    got = B.beam_select(x, score, 8, 16, out=out, ws=ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(a is b for a, b in zip(got, out))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.beam_select(x, score, 8, 16, ws=ws)
    for i in range(4):
        x.copy_(draw(50 + i, 16, 30000, "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in got]
        assert all(torch.equal(a, b) for a, b in zip(kept, B.beam_select(x, score, 8, 16)))


def test_refusals(B):
    x, s = torch.zeros((8, 100), device="cuda"), torch.zeros(8, device="cuda")
    with pytest.raises(TypeError):
        B.beam_select(x.double(), s, 4)
    with pytest.raises(TypeError):
        B.beam_select(x.t(), s, 4)
    with pytest.raises(ValueError):
        B.beam_select(x, s, 3)
    with pytest.raises(ValueError):
        B.beam_select(x, s, 0)
    with pytest.raises(ValueError):
        B.beam_select(x, s[:4].contiguous(), 4)
    with pytest.raises(ValueError):
        B.beam_select(x, s, 4, 65)
    with pytest.raises(ValueError):
        B.beam_select(x[:1].expand(8, 100), s, 4)
    with pytest.raises(TypeError):
        B.beam_select(x, s.double(), 4)
    with pytest.raises(TypeError):
        B.beam_select(x, s, 4, done=s)
    with pytest.raises(Exception):
        B.beam_select(x, s, 4, done=torch.zeros(8, dtype=torch.int32, device="cuda"), end=100)
    with pytest.raises(ValueError):
        out = B.beam_select(x, s, 4)
        B.beam_select(x, s, 4, 5, out=out)


def test_empty(B):
    x, s = torch.zeros((0, 100), device="cuda"), torch.zeros(0, device="cuda")
    parent, token, score = B.beam_select(x, s, 4)
    assert parent.shape == token.shape == score.shape == (0, 4)
