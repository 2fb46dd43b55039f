"""symph_beam_select against its definition in 64 bits: sizes, widths, ties, masks, ended beams, addresses."""
import numpy as np
import pytest
import torch

import beam_ref as R
import paper_2412_16434_amd as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")
LEFT = 77  # what outputs hold before a call


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).to(DEV)


def _starts(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(int)


def _call(logits, scores, cu, cu_next, max_next, end, rows_of_ends=True, behind=3, **kw):
    """The call's outputs as numpy; `behind`: entries behind the last session's, which have to be left alone."""
    total = int(cu_next[-1]) + behind
    parents, tokens = _i32(np.full(total, LEFT)), _i32(np.full(total, LEFT))
    best = torch.full((total,), float(LEFT), device=DEV)
    ends = torch.full((logits.shape[0],), float(LEFT), device=DEV) if rows_of_ends else None
    size = S.beam_select_workspace_bytes(*logits.shape, max_next)
    space = torch.full((max(size, 1),), 255, dtype=torch.uint8, device=DEV)
    S.beam_select(logits, torch.as_tensor(scores, dtype=torch.float32).to(DEV), _i32(cu), _i32(cu_next), max_next, parents, tokens, best,
                  end_token=end, end_scores=ends, workspace=space, **kw)
    torch.cuda.synchronize()
    return dict(parents=parents.cpu().numpy(), tokens=tokens.cpu().numpy(), next_scores=best.cpu().numpy(),
                end_scores=None if ends is None else ends.cpu().numpy())


def _check(logits, scores, beams, widths, end=-1, max_next=None, **kw):
    cu, cu_next = _starts(beams), _starts(widths)
    max_next = max(widths) if max_next is None else max_next
    got = _call(logits, scores, cu, cu_next, max_next, end, **kw)
    want = R.beam_select(logits.float().cpu().numpy(), np.asarray(scores, np.float32), cu, cu_next, max_next, end)
    n, rows = int(cu_next[-1]), int(cu[-1])
    for name in ("parents", "tokens"):
        assert np.array_equal(got[name][:n], want[name]), (name, got[name][:n], want[name])
        assert np.all(got[name][n:] == LEFT)
    _near(got["next_scores"][:n], want["next_scores"], want["tol"])
    assert np.all(got["next_scores"][n:] == LEFT)
    if got["end_scores"] is not None:
        _near(got["end_scores"][:rows], want["end_scores"][:rows], want["end_tol"][:rows])
        assert np.all(got["end_scores"][rows:] == LEFT)


def _near(got, want, tol):
    there = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), there) and np.all(got[~there] == -INF)
    off = np.abs(got[there].astype(np.float64) - want[there])
    assert np.all(off <= tol[there]), (off.max(), tol[there][off.argmax()])


def _normal(rows, vocab, dtype, seed, scale=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((rows, vocab), generator=g) * scale).to(dtype).to(DEV)


def _scores(rows, seed):
    return np.random.RandomState(seed).uniform(-9, -1, rows).astype(np.float32)


BF16, FP32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("vocab", [1, 2, 7, 63, 64, 65, 511, 513, 2047, 2049, 8191, 8193, 16385, 50001, 131072])
def test_sizes_of_the_vocabulary(vocab, dtype):
    _check(_normal(9, vocab, dtype, vocab), _scores(9, vocab), [4, 2, 3], [4, 5, 1], end=vocab // 2)


@pytest.mark.parametrize("vocab,width", [(1_300_007, 5), (3_000_001, 64), (3_000_001, 1)])
def test_rows_of_more_than_64_parts(vocab, width):
    _check(_normal(2, vocab, BF16, width), _scores(2, 5), [2], [width], end=7)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("beams,widths", [([1], [1]), ([1], [64]), ([64], [64]), ([64, 1, 0, 3], [3, 0, 5, 64]), ([0], [4]),
                                          ([130], [17]), ([300, 2], [9, 3]), ([1] * 70, [2] * 70), ([5, 0, 0, 5], [33, 0, 1, 31])])
def test_widths_of_sessions(beams, widths, dtype):
    rows = sum(beams)
    _check(_normal(max(rows, 1), 5003, dtype, rows), _scores(max(rows, 1), 3), beams, widths, end=17)


@pytest.mark.parametrize("seed", range(6))
def test_random_batches(seed):
    rs = np.random.RandomState(seed)
    beams = rs.randint(0, 13, size=rs.randint(1, 20)).tolist()
    widths = rs.randint(0, 25, size=len(beams)).tolist()
    widths[0] = max(widths[0], 1)
    rows, vocab = max(sum(beams), 1), int(rs.randint(1, 40000))
    logits = _normal(rows, vocab, BF16 if seed % 2 else FP32, seed)
    logits.masked_fill_(torch.rand(logits.shape, generator=torch.Generator().manual_seed(seed)).to(DEV) < rs.choice([0.0, 0.5, 0.999]), -INF)
    scores = np.where(rs.random_sample(rows) < 0.2, -np.inf, _scores(rows, seed))
    _check(logits, scores, beams, widths, end=int(rs.randint(-1, vocab)))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("width", [1, 6, 64])
def test_equal_values_go_to_the_lowest(dtype, width):
    """All logits of a row equal, rows equal: beams, then tokens, in order; zeros of both signs are equal."""
    logits = torch.zeros((3, 9001), dtype=dtype, device=DEV)
    logits[:, ::2] = -0.0
    _check(logits, [-1.0, -1.0, -1.0], [3], [width], end=0)
    logits[1] = 0.5
    _check(logits, [-1.0, -1.0, -1.0], [3], [width])


@pytest.mark.parametrize("vocab", [999, 8193, 30001])
def test_equal_beams_tie_wherever_their_rows_begin(vocab):
    """Copies of a row at addresses of every alignment: equal sums, so the lower beam comes first."""
    row = _normal(1, vocab, BF16, 5)
    _check(row.expand(8, vocab).contiguous(), [-2.0] * 8, [8], [64])


@pytest.mark.parametrize("order", ["rising", "falling", "late peak", "steps"])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_orders_that_fill_every_list(order, dtype):
    vocab = 40000
    x = torch.arange(vocab, dtype=torch.float32) / 4000
    x = {"rising": x, "falling": x.flip(0), "late peak": torch.where(torch.arange(vocab) >= vocab - 70, x, torch.zeros(())),
         "steps": torch.floor(x)}[order]
    _check(x.to(dtype).to(DEV).expand(4, vocab).contiguous(), [-1.0, -1.5, -0.5, -1.0], [4], [64], end=vocab - 1)


@pytest.mark.parametrize("rows,tiles", [(512, 16), (820, 8), (1366, 3), (2049, 2)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_tokens_that_wait_while_the_last_tiles_have_none(rows, tiles, dtype):
    """Forty tokens in every tile of the first half, in as many lanes, and nothing behind: all waves bring theirs to the end at once."""
    logits = torch.full((rows, tiles * 2048), -INF)
    per = 8 if dtype == BF16 else 4                     # neighbouring values of a lane
    rs = np.random.RandomState(rows)
    for tile in range((tiles + 1) // 2):
        tokens = tile * 2048 + (np.arange(40) + 8 * tile) % 64 * per
        logits[:, tokens] = torch.from_numpy(rs.standard_normal((rows, 40)).astype(np.float32))
    _check(logits.to(dtype).to(DEV), _scores(rows, 4), [1] * rows, [64] * rows, end=(per * 3) % 64)


@pytest.mark.parametrize("rows,waves", [(512, 8), (820, 4), (1366, 2), (2049, 1)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_equal_values_that_are_looked_at_late(rows, waves, dtype):
    """A wave's second tile has three tokens (few: they are looked at together with later ones) and its third fifty (many: at once), all of
    one value: the three come first.  In the last row another wave's tiles have the same value behind them."""
    tile = 2048
    logits = torch.full((rows, 5 * waves * tile), -INF)
    per = 8 if dtype == BF16 else 4                     # neighbouring values of a lane
    lanes = torch.arange(64) * per
    logits[:, lanes[:20]] = 1.0
    logits[:, waves * tile + lanes[[5, 9, 40]]] = 2.0
    logits[:, 2 * waves * tile + lanes[:50]] = 2.0
    logits[-1, (waves + 1) * tile + lanes[:50]] = 2.0
    _check(logits.to(dtype).to(DEV), _scores(rows, 6), [1] * rows, [8] * rows, end=waves * tile + 9 * per)


@pytest.mark.parametrize("rows,waves,beams", [(513, 7, 1), (820, 4, 4), (1366, 2, 2), (2049, 1, 3)])
@pytest.mark.parametrize("seed", range(4))
def test_few_values_and_many_tiles(rows, waves, beams, seed):
    """Tiles of a few tokens, of many and of none by chance, of values that many share, for parts of several tiles a wave."""
    rs, tile = np.random.RandomState(seed), 2048
    vocab = 6 * waves * tile + int(rs.randint(tile))
    kinds, levels = 24, int(rs.choice([1, 2, 5, 40]))
    drawn = np.full((kinds, vocab), -np.inf, np.float32)
    for k in range(kinds):
        for t in range(0, vocab, tile):
            there = rs.random_sample(min(tile, vocab - t)) < rs.choice([0, 0.0005, 0.002, 0.006, 0.02, 0.05])
            drawn[k, t:t + there.size][there] = np.floor(rs.random_sample(int(there.sum())) * levels + t * rs.choice([0, 1]) / vocab * levels)
    logits = torch.from_numpy(drawn).to(BF16 if seed % 2 else FP32).to(DEV)[torch.arange(rows, device=DEV) % kinds]
    sessions = [beams] * (rows // beams) + ([rows % beams] if rows % beams else [])
    _check(logits, rs.choice([-1.0, -2.0, -3.5], rows), sessions, rs.choice([1, 4, 9, 30, 64], len(sessions)).tolist(), end=vocab // 3)


def test_few_tokens_left():
    """Fewer candidates than are wanted: what there is, then nothing."""
    logits = torch.full((4, 3000), -INF, device=DEV)
    logits[0, 2999], logits[1, 0], logits[1, 7], logits[3, 5] = 1.0, 2.0, 2.0, -3.0
    _check(logits, [-1.0] * 4, [2, 1, 1], [5, 3, 2], end=7)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_masks_infinities_and_nan(dtype):
    lowest, highest = torch.finfo(dtype).min, torch.finfo(dtype).max
    logits = _normal(7, 4099, dtype, 9)
    logits[0, 100:4000] = lowest
    logits[1] = lowest                       # nothing but the lowest value: an even distribution
    logits[2, ::3] = float("nan")
    logits[3] = float("nan")
    logits[4, 50] = INF
    logits[4, 4050] = INF
    logits[5, 7] = highest
    logits[6] = -INF
    _check(logits, [-1.0] * 7, [1] * 7, [9] * 7, end=3)
    _check(logits, [-1.0] * 7, [7], [60], end=50)


def test_beams_that_have_ended_are_not_read():
    """Scores that are not finite: no candidates, whatever the logits hold."""
    logits = _normal(5, 3001, FP32, 2)
    logits[1] = float("nan")
    _check(logits, [-1.0, -np.inf, np.nan, np.inf, -2.0], [5], [8], end=11)
    _check(logits, [-np.inf] * 5, [3, 2], [4, 4], end=11)


def test_end_tokens_among_the_best():
    """The end token is the best of some beams, the last that still counts of others, one too many of others."""
    logits = _normal(6, 2000, FP32, 4, scale=1.0)
    logits[:, 5] = torch.tensor([9.0, 4.2, 3.5, 3.0, 2.5, -9.0]).to(DEV)
    for width in (1, 2, 3, 4, 7, 20):
        _check(logits, np.linspace(-1, -2, 6), [6], [width], end=5)
    _check(logits, np.linspace(-1, -2, 6), [6], [4], end=5, rows_of_ends=False)
    _check(logits, np.linspace(-1, -2, 6), [6], [4], end=-1)


@pytest.mark.parametrize("first,stride", [(0, 3333), (1, 3334), (3, 3339), (8, 3400)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_rows_at_any_address(first, stride, dtype):
    whole = torch.full((5, stride), INF, dtype=dtype, device=DEV)   # (values beside the rows would win)
    logits = whole[:, first:first + 3325]
    logits.copy_(_normal(5, 3325, dtype, first))
    _check(logits, _scores(5, 1), [3, 2], [4, 4], end=9)


def test_rows_and_sessions_that_do_not_fit():
    """Offsets past the rows or the entries are cut there; rows of no session and entries past max_next."""
    logits = _normal(6, 1000, FP32, 8)
    got = _call(logits, [-1.0] * 6, np.array([0, 2, 4]), np.array([0, 5, 7]), 3, 1)
    want = R.beam_select(logits.cpu().numpy(), np.full(6, -1.0), [0, 2, 4], [0, 5, 7], 3, 1)
    assert np.array_equal(got["tokens"][:7], want["tokens"]) and np.array_equal(got["tokens"][3:5], [-1, -1])
    assert np.all(got["end_scores"][4:] == LEFT) and np.all(got["tokens"][7:] == LEFT)
    got = _call(logits, [-1.0] * 6, np.array([-3, 2, 90]), np.array([0, 3, 6]), 3, 1, behind=0)
    want = R.beam_select(logits.cpu().numpy(), np.full(6, -1.0), [0, 2, 6], [0, 3, 6], 3, 1)
    assert np.array_equal(got["tokens"], want["tokens"]) and np.array_equal(got["parents"], want["parents"])


def test_scores_far_from_zero():
    logits = _normal(4, 7000, FP32, 3)
    _check(logits + 3e4, [-1e5, -1e5, -1e5, -2e5], [4], [8], end=2)
    _check(logits * 1e-6, [-1e-3, -1e-3, -1.0, -2e-3], [4], [8], end=2)


def test_two_calls_at_once_and_again():
    """Two streams with workspaces of their own; the same call twice gives the same bits."""
    logits, scores = _normal(64, 30001, BF16, 12), _scores(64, 12)
    cu = _starts([8] * 8)
    one = _call(logits, scores, cu, cu, 8, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        two = _call(logits, scores, cu, cu, 8, 3)
    three = _call(logits, scores, cu, cu, 8, 3, stream=torch.cuda.current_stream())
    for name in one:
        assert np.array_equal(one[name], two[name]) and np.array_equal(one[name], three[name])
