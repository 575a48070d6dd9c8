"""Decoding over a paged cache where it can go wrong: probabilities that fp16 barely holds, scores that fp32 barely holds, infinities, NaN, pages and
lengths outside the pages, in every form of the attention (rows of a key head: 16, 32, 64, 128, 256; pages by TMA and by cp.async); what a
status word keeps."""
import math

import pytest
import torch

from test_gpu_paged_ops import BF16, FP16, check_attention, jot, normal, pool, spread  # noqa: F401 (jot: the fixture)

pytestmark = pytest.mark.gpu

ROWS = [5, 20, 40, 80, 150]                # one of each tile of rows, with one query head a key head
PAGES = [16, 24, 10]                       # whole tiles by TMA, tiles of 120 keys by TMA, by cp.async


def int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------------------------- status words
def test_a_bad_index_does_not_take_an_expired_wait_off_the_record(jot):
    """2 says that outputs are undefined: an index that is reported after it must not make a mere bad index of it."""
    for page in (16, 10):
        pages, table = spread(jot, 5, [100], 2, page, 64, BF16)
        x, outside = normal(1, (1, 2, 64), BF16), int32([pages.n_pages * page])
        freq = jot.rope_frequencies(64, 1e4)
        broken = table.clone()
        broken[0, 1] = pages.n_pages

        def attend(T, t, n):
            return lambda s: jot.paged_attention(normal(2, (1, T, 2, 64), BF16), pages, t.cuda(), int32([n]), status=s)

        calls = [lambda s: jot.kv_write(pages, x, x, outside, status=s),
                 lambda s: jot.head_norm_rope(x, x, int32([3]), jot.Rope(freq), v=x, pages=pages, slots=outside, status=s)]
        calls += [attend(T, broken, 100) for T in ROWS] + [attend(T, table[:, :2], 100) for T in ROWS]
        for call in calls:
            for held, want in ((0, jot.STATUS_BAD_INDEX), (2, 2), (jot.STATUS_BAD_INDEX, jot.STATUS_BAD_INDEX)):
                status = int32([held])
                call(status)
                assert int(status) == want


# ---------------------------------------------------------------------------------------------- numerics
@pytest.mark.parametrize("page", [64, 10])
@pytest.mark.parametrize("T,n", [(5, 2 ** 19), (20, 2 ** 19), (40, 2 ** 18), (80, 2 ** 17), (150, 2 ** 17)])
def test_a_long_flat_tail_beside_one_key_that_leads(jot, T, n, page):
    """One key in front of hundreds of thousands that each weigh just under 2^-25 of it, and 0.4 % to 1.6 % together: fp16's smallest number
    is 2^-24, so that weights taken relative to the leading one vanish from the product while the sum counts them.  The leading value is 0
    and the others 1: what comes out is the others' share.  As many sequences (over the same pages) as there are shares of the work, so
    that none is cut into parts with maxima of their own; a warp's range of keys, or a copy of a row, has 2^17 of them."""
    hd, seqs, lead_by = 64, 448, 25.0625
    n_pages = (n + page - 1) // page
    pages = jot.KVPages(torch.zeros(1, n_pages, 1, page, hd, dtype=FP16, device="cuda"), torch.ones(1, n_pages, 1, page, hd, dtype=FP16, device="cuda"))
    q = torch.zeros(1, T, 1, hd, dtype=FP16, device="cuda")
    q[..., 0] = 16
    q, table, lens = q.expand(seqs, -1, -1, -1), torch.arange(n_pages, dtype=torch.int32, device="cuda")[None].expand(seqs, -1), int32([n] * seqs)
    for lead in (0, n // 2 + 7):
        pages.k.zero_()
        pages.v.fill_(1)
        pages.k[0, lead // page, 0, lead % page, 0] = lead_by / 16          # exact in fp16
        pages.v[0, lead // page, 0, lead % page] = 0
        lse = torch.empty(seqs, T, 1, device="cuda")
        out = jot.paged_attention(q, pages, table, lens, scale=math.log(2), lse=lse)
        tail = (n - 1) * 2.0 ** -lead_by
        # The result's rounding: 2^-11.  A weight's: with the leading one at 2^7 the others are 2^-18.1, of which half of 2^-24 is 2^-6.9.  The sum,
        # in fp32 beside the leading weight: every pair of the thread that has the leading key, half an ulp at each of 2^14 steps, 2^-10; the
        # product's own sum holds nothing but such weights, with an ulp of 2^-23 lost at each of 2^13 steps of 16 keys: 2^-10
        err = (out.double() - tail / (1 + tail)).abs().max().item()
        assert err <= (2.0 ** -11 + 2.0 ** -6.9 + 2.0 ** -10 + 2.0 ** -10) * tail, (lead, err / tail)
        want = lead_by * math.log(2) + math.log1p(tail)
        assert ((lse.double() - want).abs() <= 2.0 ** -10 + 2.0 ** -20 + 2.0 ** -22 * want).all()


@pytest.mark.parametrize("page", [16, 10])
@pytest.mark.parametrize("dtype,size", [(FP16, 4000.0), (FP16, 60000.0), (BF16, 30000.0), (BF16, 2.0 ** 40)])
@pytest.mark.parametrize("T", ROWS)
def test_scores_of_which_fp32_holds_no_fraction(jot, T, dtype, size, page):
    """Scores of 10^8 and more, alike or far apart: the leading keys share the weight evenly."""
    n, hd = 300, 128
    pages, table = spread(jot, 3, [n], 1, page, hd, dtype)
    q = torch.full((1, T, 1, hd), size, dtype=dtype, device="cuda")
    ids = table[0, :(n + page - 1) // page].long().cuda()
    values = pages.v[0][ids, 0].reshape(-1, hd)[:n].double()
    for small, sign in ((0, 1), (200, 1), (200, -1)):                       # so many keys of zeros in front, whose weight is zero
        keys = torch.zeros(len(ids) * page, hd, dtype=dtype, device="cuda")
        keys[small:n] = sign * size
        pages.k[0, ids] = keys.view(len(ids), 1, page, hd)
        lse = torch.empty(1, T, 1, device="cuda")
        out = jot.paged_attention(q, pages, table.cuda(), int32([n]), scale=sign * hd ** -0.5, lse=lse)[0, :, 0].double()
        want, total = values[small:].mean(0), values[small:].abs().mean(0)
        # alike scores have alike weights, powers of two apart from the rescaling of sums: no rounding of a weight but its own
        tol = torch.finfo(dtype).eps / 2 * (want.abs() + total) + 2.0 ** -18 * total
        assert ((out - want).abs() <= tol).all(), (small, sign, out[0, :3], want[:3])
        top = float(torch.tensor(size, dtype=dtype).double() ** 2 * hd) * hd ** -0.5
        assert ((lse.double() - top).abs() <= 2.0 ** -20 * top).all()


@pytest.mark.parametrize("T", ROWS)
def test_a_scale_of_zero_gives_the_mean_of_the_values(jot, T):
    n, hd = 200, 64
    for dtype, size in ((BF16, 1.0), (FP16, 1.0), (BF16, 2.0 ** 60)):       # scores of up to 2^126, times zero
        pages, table = spread(jot, 7, [n], 1, 16, hd, dtype)
        pages.k.mul_(size)
        q = normal(9, (1, T, 1, hd), dtype) * size
        ids = table[0, :13].long().cuda()
        v = pages.v[0][ids, 0].reshape(-1, hd)[:n].double()
        lse = torch.empty(1, T, 1, device="cuda")
        for scale in (0.0, -0.0):
            out = jot.paged_attention(q, pages, table.cuda(), int32([n]), scale=scale, lse=lse)[0, :, 0].double()
            tol = torch.finfo(dtype).eps / 2 * (v.mean(0).abs() + v.abs().mean(0)) + 2.0 ** -18 * v.abs().mean(0)
            assert ((out - v.mean(0)).abs() <= tol).all()
            assert ((lse.double() - math.log(n)).abs() <= 2.0 ** -20 + 2.0 ** -22 * math.log(n)).all()


@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("T", ROWS)
def test_infinite_and_nan_scores_in_every_form(jot, T, page):
    """A NaN query, an infinite one and an infinite key element reach the rows whose scores they are, and no other."""
    n, hd = 333, 64
    for dtype in (BF16, FP16):
        pages, table = spread(jot, 11, [n, n], 1, page, hd, dtype)
        args = table.cuda(), int32([n, n])
        q = normal(13, (2, T, 1, hd), dtype)
        q[..., 0] = torch.where(q[..., 0] >= 0, 1.0, -1.0).to(dtype)
        plain = jot.paged_attention(q, pages, *args)
        # NaN and infinite queries: their rows are NaN (an infinite query meets keys of either sign), the others keep their bits
        bad = q.clone()
        bad[0, T // 2, 0, 3], bad[1, 0, 0, 0] = math.nan, math.inf
        out = jot.paged_attention(bad, pages, *args)
        hit = torch.zeros(2, T, dtype=torch.bool, device="cuda")
        hit[0, T // 2] = hit[1, 0] = True
        assert out[hit].isnan().all() and torch.equal(out[~hit], plain[~hit])
        # an infinite key element: rows with a positive query element there have a score of infinity, whose softmax is no number; for the others
        # the key does not count: as if it scored far below all others
        k, v = (t[0][table[0, :(n + page - 1) // page].long().cuda(), 0].reshape(-1, hd)[:n].double() for t in (pages.k, pages.v))
        for j in (0, 130, n - 1):
            saved = pages.k[0, table[0, j // page], 0, j % page, 0].clone()
            pages.k[0, table[0, j // page], 0, j % page, 0] = math.inf
            lse = torch.empty(2, T, 1, device="cuda")
            out = jot.paged_attention(q, pages, *args, lse=lse)
            up = q[0, :, 0, 0] > 0
            assert out[0][up].isnan().all() and not lse[0][up].isfinite().any()
            s = q[0, :, 0].double() @ k.T * hd ** -0.5
            s[:, j] = -math.inf
            p = torch.softmax(s, -1)
            eps = torch.finfo(dtype).eps
            tol = eps / 2 * ((p @ v).abs() + p @ v.abs()) + 2.0 ** -14 * (p @ v.abs()) + 2.0 ** -24
            assert ((out[0, :, 0].double() - p @ v).abs() <= tol)[~up].all()
            assert torch.equal(out[1], plain[1])
            pages.k[0, table[0, j // page], 0, j % page, 0] = saved
        # scores of minus infinity only: nothing to weigh, and the logarithm of nothing
        pages.k[0, :, 0, :, 0] = pages.k[0, :, 0, :, 0].abs().clamp(min=0.5)
        bad = q.clone()
        bad[0, 1, 0, 0] = -math.inf
        lse = torch.empty(2, T, 1, device="cuda")
        out, again = jot.paged_attention(bad, pages, *args, lse=lse), jot.paged_attention(q, pages, *args)
        hit = torch.zeros(2, T, dtype=torch.bool, device="cuda")
        hit[0, 1] = True
        assert out[hit].isnan().all() and (lse[hit] == -math.inf).all() and torch.equal(out[~hit], again[~hit])


# ---------------------------------------------------------------------------------------------- pages and lengths outside
@pytest.mark.parametrize("page", PAGES + [256])
@pytest.mark.parametrize("T", ROWS)
def test_pages_outside_the_pool_read_as_zeros_in_every_form(jot, T, page):
    lens = [700, 40]
    for hd in (64, 128):
        pages, table = spread(jot, 45, lens, 2, page, hd, BF16)
        used = set(table[table >= 0].tolist())
        blank = next(p for p in range(pages.n_pages) if p not in used)
        pages.k[0, blank] = pages.v[0, blank] = 0
        q = normal(8, (2, T, 2, hd), BF16)
        dl = int32(lens)
        for at in (0, 1, (lens[0] - 1) // page):
            t = table.clone()
            t[0, at] = blank
            want, _ = check_attention(jot, q, pages, t, lens)
            for bad in (-1, pages.n_pages, 2 ** 31 - 1, -2 ** 31):
                t[0, at] = bad
                status = int32([0])
                out = jot.paged_attention(q, pages, t.cuda(), dl, status=status)
                assert int(status) == jot.STATUS_BAD_INDEX and torch.equal(out, want)
        # a length beyond the table's row counts up to its end
        status = int32([0])
        t = table[:, :2].cuda()
        out = jot.paged_attention(q, pages, t, int32([2 ** 31 - 1, 40 if page > 20 else 2 * page]), status=status)
        assert int(status) == jot.STATUS_BAD_INDEX
        assert torch.equal(out, jot.paged_attention(q, pages, t, int32([2 * page, 40 if page > 20 else 2 * page])))


@pytest.mark.parametrize("T", ROWS)
def test_pages_that_lie_backwards(jot, T):
    """A page stride below zero (the library's interface takes it): the pool from its other end."""
    n, hd, page = 500, 64, 16
    pages, table = spread(jot, 17, [n], 2, page, hd, BF16)
    q = normal(19, (1, T, 4, hd), BF16)
    stride, last = pages.k.stride(1), pages.n_pages - 1
    turned = jot.KVPages(pages.k.flip(1).contiguous(), pages.v.flip(1).contiguous())       # what the pool is, seen from there
    turned._packed = jot._pack_pages(pages.k[0, last].data_ptr(), pages.v[0, last].data_ptr(), pages.k.stride(0), pages.v.stride(0), -stride, -stride, 1,
                                     pages.n_pages, 2, page, hd, 0)
    check_attention(jot, q, turned, torch.where(table >= 0, last - table, table), [n])
    x, slots = normal(23, (3, 4, hd), BF16), int32([0, 5 * page + 3, last * page + 1])
    jot.kv_write(turned, x[:, :2], x[:, 2:], slots)
    for r, s in enumerate(slots.tolist()):
        assert torch.equal(pages.k[0, last - s // page, :, s % page], x[r, :2]) and torch.equal(pages.v[0, last - s // page, :, s % page], x[r, 2:])


# ---------------------------------------------------------------------------------------------- workspace
@pytest.mark.parametrize("T", ROWS)
@pytest.mark.parametrize("lens", [[20011], [1, 9000, 0, 700, -1, 5], [300] * 200])
def test_what_a_workspace_holds_before_does_not_matter(jot, T, lens):
    pages, table = spread(jot, 29, lens, 1, 16, 64, BF16)
    q = normal(31, (len(lens), T, 1, 64), BF16)
    ws = torch.empty(jot.paged_attention_workspace_bytes(T, 1, 1, 64), dtype=torch.uint8, device="cuda")
    outs = []
    for fill in (0, 0xff, 0x7f, 1):
        ws.fill_(fill)
        out, lse = check_attention(jot, q, pages, table, lens, workspace=ws)
        outs.append((out.clone(), lse.clone()))
    assert all(torch.equal(a, b) for o in outs[1:] for a, b in zip(o, outs[0]))
