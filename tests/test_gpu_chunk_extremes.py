"""GPU: attention of chunks where scores are very large or no numbers, against plain 64-bit sums on the host.

Large scores: queries and keys are whole numbers times powers of two, chosen so that every dot product is a whole number
below 2^24 times one power of two: exact in 32 bits in any order.  Different scores of a row are then at least one such unit
apart, which the tests make 2^6 or more after scaling, so a row is the mean of V over the keys with the largest score (the
others' weights are below 2^-64).  Their weights are equal, and lie between 1/2 and 2^8 where the scaled score is no whole
number: rounded to bf16 (2^-8) for the product with V, not in the sum below.  What remains: exp2 (2^-19 as in the other
tests), sums over n keys (n x 2^-24 each, above and below), the quotient and its product (2^-23) and the output's rounding,
so |error| <= 2^-8 |want| + A (2^-8 + 2^-18 + n 2^-23) with A the mean of |V|."""
import math

import pytest
import torch

from test_gpu_chunk import PAGE, Case, _ragged, _say

pytestmark = pytest.mark.gpu


def _largest_scores(c, i, x):
    """Rows of chunk i as the mean of V over the keys of the largest score, and their tolerance, fp64 [n][d]."""
    n, p, _, _ = c.chunks[i]
    r0 = int(c.row0[i])
    q = x[r0:r0 + n].double().view(n, c.H, c.hd).transpose(0, 1)
    (K, _), (V, _) = c.cache(i, 0), c.cache(i, 1)
    sc = q @ K.transpose(1, 2)
    sc = sc.masked_fill(torch.arange(p + n)[None, :] > torch.arange(p, p + n)[:, None], -math.inf)
    e = (sc == sc.amax(-1, keepdim=True)).double()
    keys = e.sum(-1, keepdim=True)
    want, A = e @ V / keys, e @ V.abs() / keys
    tol = want.abs() * 2 ** -8 + A * (2 ** -8 + 2 ** -18 + keys * 2 ** -23)
    return tuple(t.transpose(0, 1).reshape(n, -1) for t in (want, tol))


def _check_largest(c, got, x):
    for i, (n, _, _, _) in enumerate(c.chunks):
        r0 = int(c.row0[i])
        want, tol = _largest_scores(c, i, x)
        err = (got[r0:r0 + n].double() - want).abs()
        assert (err <= tol).all(), (i, c.chunks[i], (err / tol).max().item())  # a NaN is not <=


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_one_key_with_a_large_score(dtype):
    """A first token sees itself alone: its row is V, whatever its score."""
    _say(f"one key {dtype}")
    for H, hd in ((4, 64), (3, 96), (2, 128)):
        for size in (64.0, 4096.0, 9984.0, 16384.0, 19968.0, 29952.0, 2.0 ** 20, 2.0 ** 40, 2.0 ** 59):
            for sign in (1, -1):
                c = Case(H, hd, [(1, 0, 0, 0)], seed=41)
                c.pool[1, :, 0] = size
                c.q[:] = sign * size
                got, q = c.device().attend(dtype)
                assert c.code() == 0
                v = c.cache(0, 1)[0][:, 0].reshape(-1)
                assert torch.equal(got[0].double(), v), (H, hd, size, sign)


# few steps, segments that are joined, tiles with steps that every row sees, ragged
LARGE = [_ragged((13, 700)), _ragged((1, 2000), (3, 64)), _ragged((300, 2100)), _ragged((128, 0), (129, 5), (33, 500), (1, 300)),
         _ragged((1100, 1000), (1024, 0))]


@pytest.mark.parametrize("chunks", LARGE, ids=str)
def test_large_scores(chunks):
    """Scores of one size and of sizes that grow along the context, units of 2^15 to 2^86.  bf16 queries: those in 32 bits are
    read in two parts, which settles which of several equal scores is the largest."""
    _say(f"large {chunks}")
    for H, hd in ((4, 64), (3, 96), (2, 128)):
        for a, b, grows in ((5, 10, 0), (8, 10, 0), (10, 13, 0), (14, 15, 1), (12, 13, 2), (40, 40, 1)):
            c = Case(H, hd, chunks, seed=42)
            g = torch.Generator().manual_seed(43)
            # sums of at most 128 products of up to 4 x 4, below 2^12 of the key's units
            x = torch.randint(-4, 5, c.q.shape, generator=g).float()
            k = torch.randint(-4, 5, c.pool[1, :, 0].shape, generator=g).float()
            if grows:
                at = torch.zeros(c.pages, PAGE)
                for i, (n, p, s, loop) in enumerate(chunks):
                    for t in range(p + n):
                        at[c.table[s, c.plane(loop), t // PAGE], t % PAGE] = t * 7 // (p + n)  # 0 to 6
                k *= (2.0 ** (at * grows))[:, None, :, None]
            c.q = x * 2.0 ** a
            c.pool[1, :, 0] = (k * 2.0 ** b).to(torch.bfloat16)
            assert torch.equal(c.pool[1, :, 0].float(), k * 2.0 ** b)
            got, q = c.device().attend()
            assert c.code() == 0
            _check_largest(c, got, q)


def test_large_scores_leave_other_rows():
    """Rows with large scores beside ordinary ones: the others keep their bits."""
    _say("other rows")
    chunks = _ragged((70, 300), (40, 0))
    for H, hd in ((4, 64), (2, 128)):
        c = Case(H, hd, chunks, seed=44)
        clean, q = c.device().attend()
        c.check(clean, q)
        big = c.q.clone()
        rows = torch.arange(c.M) % 7 == 3
        big[rows] *= 2.0 ** 40
        got, _ = c.attend(q=big)
        assert torch.equal(got[~rows], clean[~rows])
        assert torch.isfinite(got).all()


# one segment, and several that are joined
@pytest.mark.parametrize("chunks", [_ragged((13, 0)), _ragged((13, 700)), _ragged((200, 300), (1, 500))], ids=str)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_query_that_is_no_number(dtype, chunks):
    """Every score of the row is NaN, and so is the row, in however many segments; the others keep their bits."""
    _say(f"NaN query {dtype} {chunks}")
    for H, hd in ((4, 64), (3, 96), (2, 128)):
        c = Case(H, hd, chunks, seed=45)
        clean, _ = c.device().attend(dtype)
        q = c.q.clone()
        bad = torch.zeros(c.M, dtype=torch.bool)
        bad[[5, c.M - 1]] = True
        q.view(c.M, H, hd)[bad, :, 7] = math.nan
        got, _ = c.attend(dtype, q=q)
        assert c.code() == 0
        assert torch.isnan(got[bad]).all()
        assert torch.equal(got[~bad], clean[~bad])


@pytest.mark.parametrize("n", [13, 128, 300])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_first_key_that_is_no_number(dtype, n):
    """Every row sees it, the first one nothing else; 128 rows and more are cut into segments."""
    _say(f"NaN key {dtype} {n}")
    for H, hd in ((4, 64), (3, 96), (2, 128)):
        c = Case(H, hd, [(n, 0, 0, 1)], seed=46)
        c.pool[1, c.table[0, 2, 0], 0, :, 0, 5] = math.nan
        got, _ = c.device().attend(dtype)
        assert c.code() == 0
        assert torch.isnan(got).all()


@pytest.mark.parametrize("chunks", [_ragged((40, 30)), _ragged((13, 700)), _ragged((300, 900))], ids=str)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_infinite_keys(dtype, chunks):
    """A key with an infinite value: where it makes a score of +inf or NaN the row is no number; where it makes one of -inf
    the row is no number either, or what it is without the key.  Rows that do not see it keep their bits."""
    _say(f"infinite keys {dtype} {chunks}")
    (n, p, s, loop), = chunks
    for H, hd in ((4, 64), (3, 96), (2, 128)):
        for value in (math.inf, -math.inf):
            for t in (3, p + 7):
                c = Case(H, hd, chunks, seed=47)
                clean, q = c.device().attend(dtype)
                at = c.table[s, c.plane(loop), t // PAGE], t % PAGE
                K, V = c.pool[1, at[0], 0, :, at[1]], c.pool[1, at[0], 1, :, at[1]]
                K[:, 5] = value
                got, _ = c.device().attend(dtype)
                assert c.code() == 0
                first = max(0, t - p)
                assert torch.equal(got[:first], clean[:first])
                # without the key, and the tolerance that the other tests take
                (x, there), (v, _) = c.cache(0, 0), c.cache(0, 1)
                sc = q.double().view(n, H, hd).transpose(0, 1) @ torch.nan_to_num(x, 0, 0, 0).transpose(1, 2) / math.sqrt(hd)
                hide = torch.arange(p + n)[None, :] > torch.arange(p, p + n)[:, None]
                hide = hide | (torch.arange(p + n) == t)[None, :]
                w = torch.softmax(sc.masked_fill(hide, -math.inf), -1)
                want, A = w @ v, w @ v.abs()
                S = q.double().abs().view(n, H, hd).transpose(0, 1) @ torch.nan_to_num(x, 0, 0, 0).abs().transpose(1, 2)
                S = (S / math.sqrt(hd)).masked_fill(hide, 0).amax(-1, keepdim=True)
                keys = (~hide).sum(-1)[None, :, None].double()
                rounded = 2 ** -16 + S * 2 ** -15 if dtype == torch.float32 else 2 ** -8 + S * 2 ** -16
                tol = want.abs() * 2 ** -8 + A * (rounded + 2 ** -19 + keys * 2 ** -23)
                near = ((got.view(n, H, hd).double() - want.transpose(0, 1)).abs() <= tol.transpose(0, 1)).all(-1)
                none = ~torch.isfinite(got.view(n, H, hd)).any(-1)
                minus = q.view(n, H, hd)[:, :, 5].float() * value == -math.inf
                assert (none | (near & minus))[first:].all(), (H, hd, value, t)
