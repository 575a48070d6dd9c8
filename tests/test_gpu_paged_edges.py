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
