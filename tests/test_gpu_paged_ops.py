"""Decoding over a paged key-value cache: every operator against its definition in float64.

Tolerances count roundings.  One rounding to an element type with `eps = torch.finfo(t).eps` is off by at most eps / 2 of the
value; below the smallest normal number by half the smallest subnormal.  A product of n terms accumulated in fp32 is off by at
most (n + 2) 2^-24 times the sum of the terms' sizes.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16
TINY = {BF16: 0.0, FP16: 2.0 ** -25}       # half of fp16's smallest subnormal; bf16's is far below anything here


@pytest.fixture(scope="module")
def jot():
    from paper_2602_11133_b200 import jot as binding
    binding._lib()
    return binding


def normal(seed, shape, dtype, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).cuda()


def pool(jot, seed, layers, n_pages, nkv, page, hd, dtype, joined=False):
    """A pool of random pages; joined: keys and values of a page beside each other in one tensor."""
    if joined:
        both = normal(seed, (layers, n_pages, 2, nkv, page, hd), dtype)
        return jot.KVPages(both[:, :, 0], both[:, :, 1])
    return jot.KVPages(normal(seed, (layers, n_pages, nkv, page, hd), dtype), normal(seed + 1, (layers, n_pages, nkv, page, hd), dtype))


# ---------------------------------------------------------------------------------------------- norm and rotation
def rope_wanted(x, positions, inv_freq, interleaved, magnitude, gain, eps):
    """(result, size of the pair each element belongs to), float64."""
    x = x.double().cpu()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double().cpu()
    half = inv_freq.numel()
    t = positions.double().cpu()[:, None, None] * inv_freq.double().cpu()
    c, s = t.cos() * magnitude, t.sin() * magnitude
    ia = torch.arange(half) * 2 if interleaved else torch.arange(half)
    ib = ia + 1 if interleaved else ia + half
    out, size = x.clone(), x.abs()
    out[..., ia], out[..., ib] = x[..., ia] * c - x[..., ib] * s, x[..., ib] * c + x[..., ia] * s
    size[..., ia] = size[..., ib] = torch.hypot(x[..., ia], x[..., ib]) * abs(magnitude)
    return out, size


def assert_heads(got, want, size, dtype):
    # one rounding to the type; before it, in fp32: angle reduced to 2^-24 turns (4e-7), sincospif, two products and a sum,
    # and the norm's mean and root (256 squares: 1e-6) -- below 4e-6 of the pair's size together
    tol = torch.finfo(dtype).eps / 2 * want.abs() + (1 + torch.finfo(dtype).eps) * 4e-6 * size + TINY[dtype]
    err = (got.double().cpu() - want).abs()
    assert (err <= tol).all(), (err / tol).max()


ROPE_CASES = [
    # rows, nq, nkv, hd, rotary, interleaved, dtype, norm, first position, magnitude
    (1, 1, 1, 64, 64, False, BF16, False, 0, 1.0),
    (1, 28, 4, 128, 128, False, BF16, True, 1_000_003, 1.1),
    (7, 4, 2, 64, 32, False, FP16, True, 17, 1.0),
    (7, 4, 2, 64, 32, True, FP16, True, 17, 0.5),
    (33, 3, 1, 128, 16, False, BF16, True, 131_000, 1.0),
    (33, 3, 1, 128, 8, True, BF16, False, 131_000, 1.0),
    (5, 2, 1, 80, 80, False, BF16, True, 3, 1.0),       # a head of ten vectors: five lanes of eight
    (5, 2, 1, 72, 64, False, BF16, True, 3, 1.0),       # an odd number of vectors
    (5, 2, 1, 72, 72, True, FP16, True, 3, 1.0),
    (5, 2, 1, 8, 8, True, FP16, True, 3, 1.0),
    (5, 2, 1, 24, 16, False, FP16, True, 3, 1.0),
    (3, 5, 5, 256, 256, False, FP16, True, 9, 1.0),
    (3, 5, 5, 192, 64, True, BF16, True, 9, 1.0),
    (4, 2, 2, 64, 0, False, BF16, True, 9, 1.0),        # no rotation: the norm alone
    (2500, 32, 8, 128, 128, False, BF16, True, 5, 1.0), # several rows a CTA, the last CTA not full
    (2501, 4, 4, 64, 64, True, FP16, True, 5, 1.0),
]


@pytest.mark.parametrize("rows,nq,nkv,hd,rotary,interleaved,dtype,norm,first,magnitude", ROPE_CASES)
def test_head_norm_rope(jot, rows, nq, nkv, hd, rotary, interleaved, dtype, norm, first, magnitude):
    # queries and keys as slices of a projection's output, whose rows are wider than the heads
    qkv = normal(1, (rows, nq + 2 * nkv, hd), dtype)
    q, k = qkv[:, :nq], qkv[:, nq:nq + nkv]
    positions = (torch.arange(rows, dtype=torch.int32) * 3 + first).cuda()
    freq = jot.rope_frequencies(rotary, 500000.0, 4.0, 8192) if rotary else torch.empty(0, device="cuda")
    gq, gk = ((1 + 0.2 * normal(2 + i, (hd,), torch.float32)).to(dtype) for i in range(2)) if norm else (None, None)
    rope = jot.Rope(freq, interleaved, magnitude)
    before = qkv.clone()
    q_out, k_out = jot.head_norm_rope(q, k, positions, rope, gq, gk, 1e-5)
    assert torch.equal(qkv, before)
    assert_heads(q_out, *rope_wanted(q, positions, freq, interleaved, magnitude, gq, 1e-5), dtype)
    assert_heads(k_out, *rope_wanted(k, positions, freq, interleaved, magnitude, gk, 1e-5), dtype)
    # in place, and with queries alone: the same bits
    jot.head_norm_rope(q, k, positions, rope, gq, gk, 1e-5, q_out=q, k_out=k)
    assert torch.equal(q, q_out) and torch.equal(k, k_out) and torch.equal(qkv[:, nq + nkv:], before[:, nq + nkv:])
    alone, none = jot.head_norm_rope(before[:, :nq], None, positions, rope, gq, eps=1e-5)
    assert none is None and torch.equal(alone, q_out)


@pytest.mark.parametrize("hd,nkv,page,joined,dtype", [(128, 4, 16, False, BF16), (64, 2, 24, True, FP16), (128, 1, 1, False, FP16),
                                                      (64, 4, 100, True, BF16), (80, 2, 7, False, BF16)])
def test_head_norm_rope_into_pages(jot, hd, nkv, page, joined, dtype):
    rows, nq, n_pages = 77, 2 * nkv, 77 // page + 9
    qkv = normal(3, (rows, nq + 2 * nkv, hd), dtype)
    q, k, v = qkv.split([nq, nkv, nkv], 1)
    pages = pool(jot, 5, 3, n_pages, nkv, page, hd, dtype, joined)
    k0, v0 = pages.k.clone(), pages.v.clone()
    slots = torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(1))[:rows].int()
    slots[5] = -1                                           # written nowhere, its query is rotated all the same
    positions = torch.arange(rows, dtype=torch.int32) + 1000
    positions[9] = -4                                       # padding: neither query nor pages are touched
    freq = jot.rope_frequencies(hd // 16 * 16, 10000.0)
    gain = (1 + 0.2 * normal(8, (hd,), torch.float32)).to(dtype)
    q_out = torch.full((rows, nq, hd), 7.0, dtype=dtype, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    back = jot.head_norm_rope(q, k, positions.cuda(), jot.Rope(freq), gain, gain, q_out=q_out, v=v, pages=pages, layer=1,
                              slots=slots.cuda(), status=status)
    assert back[0] is q_out and back[1] is None and int(status) == 0
    want, size = rope_wanted(q, positions, freq, False, 1.0, gain, 1e-6)
    live = torch.arange(rows) != 9
    assert_heads(q_out[live.cuda()], want[live], size[live], dtype)
    assert (q_out[9] == 7.0).all()
    k_alone = jot.head_norm_rope(k, None, positions.clamp(min=0).cuda(), jot.Rope(freq), gain)[0]
    for r in range(rows):
        if r not in (5, 9):
            k0[1, slots[r] // page, :, slots[r] % page] = k_alone[r]
            v0[1, slots[r] // page, :, slots[r] % page] = v[r]
    assert torch.equal(pages.k, k0) and torch.equal(pages.v, v0)        # and nothing else, in no layer


# ---------------------------------------------------------------------------------------------- pages
@pytest.mark.parametrize("rows,nkv,hd,page,joined,dtype", [(1, 1, 64, 16, False, BF16), (333, 4, 128, 24, True, BF16), (1, 32, 128, 1, False, FP16),
                                                           (2600, 2, 64, 100, False, FP16), (50, 3, 8, 5, True, BF16)])
def test_kv_write(jot, rows, nkv, hd, page, joined, dtype):
    n_pages = rows // page + 4
    pages = pool(jot, 5, 2, n_pages, nkv, page, hd, dtype, joined)
    k0, v0 = pages.k.clone(), pages.v.clone()
    kv = normal(6, (rows, 2 * nkv, hd), dtype)
    slots = torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(2))[:rows].int()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    skipped = set()
    if rows > 10:
        slots[3], slots[7] = -1, n_pages * page             # padding; outside the pages
        skipped = {3, 7}
    jot.kv_write(pages, kv[:, :nkv], kv[:, nkv:], slots.cuda(), layer=1, status=status)
    keep = torch.tensor([r for r in range(rows) if r not in skipped])
    s = slots[keep].long().cuda()
    k0[1][s // page, :, s % page] = kv[keep.cuda(), :nkv]
    v0[1][s // page, :, s % page] = kv[keep.cuda(), nkv:]
    assert torch.equal(pages.k, k0) and torch.equal(pages.v, v0)
    assert int(status) == (jot.STATUS_BAD_INDEX if skipped else 0)


@pytest.mark.parametrize("n,layers,nkv,hd,page,joined", [(1, 1, 1, 64, 1, False), (5, 3, 4, 128, 16, True), (16, 2, 2, 64, 24, False), (17, 1, 3, 8, 7, True),
                                                         (1500, 2, 1, 64, 3, False)])
def test_kv_copy_pages(jot, n, layers, nkv, hd, page, joined):
    pages = pool(jot, 9, layers, 2 * n + 3, nkv, page, hd, BF16, joined)
    k0, v0 = pages.k.clone(), pages.v.clone()
    order = torch.randperm(2 * n + 3, generator=torch.Generator().manual_seed(3)).tolist()
    src, dst = order[:n], order[n:2 * n]
    if n > 4:
        src[1] = src[0]                                     # one page onto two others
    jot.kv_copy_pages(pages, src, dst)
    src.clear()                                             # the lists were read before the call returned
    order = torch.randperm(2 * n + 3, generator=torch.Generator().manual_seed(3)).tolist()
    src = order[:n]
    if n > 4:
        src[1] = src[0]
    k0[:, dst], v0[:, dst] = k0[:, src], v0[:, src]
    assert torch.equal(pages.k, k0) and torch.equal(pages.v, v0)


def test_offsets_beyond_32_bits(jot):
    """A pool of more than 2^32 elements: the last pages are written, moved and read at 64-bit offsets."""
    page, nkv, hd = 64, 1, 128
    n_pages = 2 ** 32 // (page * nkv * hd * 2) + 7          # keys and values of a page side by side
    both = torch.empty((1, n_pages, 2, nkv, page, hd), dtype=BF16, device="cuda")
    pages = jot.KVPages(both[:, :, 0], both[:, :, 1])
    assert pages.k.stride(1) * (n_pages - 1) > 2 ** 32
    last = n_pages - 1
    kv = normal(1, (page, 2, hd), BF16)
    slots = (torch.arange(page) + last * page).int().cuda()
    jot.kv_write(pages, kv[:, :1], kv[:, 1:], slots)
    assert torch.equal(pages.k[0, last, 0], kv[:, 0]) and torch.equal(pages.v[0, last, 0], kv[:, 1])
    jot.kv_copy_pages(pages, [last], [last - 1])
    assert torch.equal(pages.k[0, last - 1, 0], kv[:, 0]) and torch.equal(pages.v[0, last - 1, 0], kv[:, 1])
    for T in (1, 40, 150):
        q = normal(2, (1, T, 2, hd), BF16)
        check_attention(jot, q, pages, torch.tensor([[last, last - 1]], dtype=torch.int32), [100])


# ---------------------------------------------------------------------------------------------- attention
def check_attention(jot, q, pages, table, lens, layer=0, scale=None, out=None, **kw):
    """Against the definition, row by row of the batch; returns (out, lse)."""
    dtype, dev = q.dtype, q.device
    B, T, nq, hd = q.shape
    group, page, eps = nq // pages.n_kv_heads, pages.page_size, torch.finfo(q.dtype).eps
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    out = torch.full(q.shape, 7.0, dtype=dtype, device=dev) if out is None else out
    lse = torch.full((B, T, nq), 7.0, device=dev)
    got = jot.paged_attention(q, pages, table.cuda(), torch.tensor(lens, dtype=torch.int32, device=dev), layer, scale, out=out, lse=lse,
                              status=status, **kw)
    assert got is out and int(status) == 0
    sc = hd ** -0.5 if scale is None else scale
    for b in range(B):
        n = lens[b]
        if n < 0:
            assert (out[b] == 7.0).all() and (lse[b] == 7.0).all()
            continue
        if n == 0:
            assert (out[b] == 0.0).all() and (lse[b] == -math.inf).all()
            continue
        ids = table[b, :(n + page - 1) // page].long().cuda()
        k, v = (t[layer][ids].permute(1, 0, 2, 3).reshape(pages.n_kv_heads, -1, hd)[:, :n].double() for t in (pages.k, pages.v))
        qq = q[b].double().view(T, pages.n_kv_heads, group, hd).permute(1, 0, 2, 3).reshape(pages.n_kv_heads, T * group, hd)
        s = qq @ k.transpose(1, 2) * sc
        p = torch.softmax(s, -1)
        want, size = p @ v, p @ v.abs()
        # a score is a product of hd terms in fp32, scaled once: off by at most `ds`, a probability by twice that, relatively
        ds = (qq.abs() @ k.abs().transpose(1, 2)).amax(-1, keepdim=True) * abs(sc) * (hd + 3) * 2.0 ** -24
        # roundings of the probabilities and of the result; sums over n keys in fp32, with two-ulp exponentials
        tol = eps / 2 * (want.abs() + size) + (2 * ds + (64 + 8) * 2.0 ** -24 + 2.0 ** -21) * size
        tol = tol + TINY[dtype] * (1 + p.amax(-1, keepdim=True) * v.abs().sum(1, keepdim=True))
        back = lambda t: t.view(pages.n_kv_heads, T, group, -1).permute(1, 0, 2, 3).reshape(T, nq, -1)
        err = (out[b].double() - back(want)).abs()
        assert (err <= back(tol)).all(), (b, n, (err / back(tol)).max().item())
        want_lse = torch.logsumexp(s, -1, keepdim=True)
        err = (lse[b].double()[..., None] - back(want_lse)).abs()
        assert (err <= back(ds) + 2.0 ** -20 + 2.0 ** -22 * back(want_lse).abs()).all(), (b, n, err.max().item())
    return out, lse


def spread(jot, seed, lens, nkv, page, hd, dtype, width=None, joined=False, layers=1):
    """A pool and a table whose sequences lie in it page by page, in no order; entries past a sequence's end are -1."""
    counts = [max(0, (n + page - 1) // page) for n in lens]
    width = max(counts + [1]) + 1 if width is None else width
    ids = torch.randperm(sum(counts) + 3, generator=torch.Generator().manual_seed(seed)).tolist()
    table, at = torch.full((len(lens), width), -1, dtype=torch.int32), 0
    for b, c in enumerate(counts):
        table[b, :c] = torch.tensor(ids[at:at + c], dtype=torch.int32)
        at += c
    return pool(jot, seed, layers, len(ids), nkv, page, hd, dtype, joined), table


ATTENTION_CASES = [
    # T, nq, nkv, hd, page, dtype, lengths
    (1, 1, 1, 64, 16, BF16, [1]),
    (1, 4, 2, 64, 16, BF16, [0, 1, 63, 64, 65, -1, 128, 129]),
    (1, 28, 4, 128, 24, FP16, [200, 0, 1, 777]),
    (1, 32, 32, 128, 64, BF16, [130, 1000]),
    (1, 28, 4, 128, 64, BF16, [20011]),                     # one sequence over every SM
    (2, 28, 4, 128, 1, BF16, [5, 70, 300]),                 # 14 rows a key head, pages of one key
    (3, 32, 4, 64, 3, FP16, [64, 191, 2, 0]),               # 24 rows
    (32, 4, 4, 64, 100, BF16, [96, 33, 0, 250]),            # 32 rows
    (33, 2, 2, 128, 16, BF16, [300, 15]),                   # one row more than a tile of 32
    (32, 28, 4, 128, 24, FP16, [400, 1, 1303]),             # 224 rows, several row tiles
    (70, 8, 2, 64, 48, BF16, [70, 500, -3]),
    (130, 2, 1, 128, 128, BF16, [513, 64]),
    (5, 5, 1, 128, 7, FP16, [1, 2, 3, 4, 5, 6, 7, 8]),
    (1, 8, 1, 64, 16, BF16, [(i * 37) % 300 - 5 for i in range(301)]),      # more sequences than a CTA has threads
    (20, 8, 8, 128, 32, FP16, [(i * 53) % 400 for i in range(40)]),
    (40, 4, 2, 64, 10, BF16, [300, 128, 129, 0]),           # pages of no multiple of eight keys: 80 and 192 rows
    (64, 6, 2, 128, 100, FP16, [450, 3]),
    (20, 4, 4, 128, 256, BF16, [700, 256, 255, 1]),         # pages larger than a tile
    (150, 2, 1, 64, 256, FP16, [1025, 130]),
    (50, 2, 2, 128, 8, BF16, [333, 128, 120, 121]),         # sixteen pages a tile
    (33, 2, 2, 64, 56, FP16, [112, 113, 500]),              # tiles of two pages with room behind them
    (18, 1, 1, 128, 120, BF16, [121, 240]),
    (20, 4, 4, 64, 200, BF16, [401, 77]),
    (1, 8, 2, 128, 16, BF16, [(i * 29) % 190 - 3 for i in range(100)]),     # tables of few tiles: sequences are not cut
    (40, 8, 2, 64, 64, BF16, [(i * 71) % 250 for i in range(50)]),
]


@pytest.mark.parametrize("T,nq,nkv,hd,page,dtype,lens", ATTENTION_CASES)
def test_paged_attention(jot, T, nq, nkv, hd, page, dtype, lens):
    pages, table = spread(jot, 21, lens, nkv, page, hd, dtype)
    q = normal(4, (len(lens), T, nq, hd), dtype)
    out, lse = check_attention(jot, q, pages, table, lens)
    again, lse2 = check_attention(jot, q, pages, table, lens)
    assert torch.equal(out, again) and torch.equal(lse, lse2)           # the same bits every time


@pytest.mark.parametrize("T,hd,dtype", [(1, 128, BF16), (40, 64, FP16), (150, 128, BF16)])
def test_paged_attention_strides_layers_and_garbage(jot, T, hd, dtype):
    """Queries and outputs inside wider tensors, keys and values interleaved, another layer, a wide table of which a slice is
    passed; whatever lies behind a length, NaN and infinities too, and in other pages, changes nothing."""
    lens, nkv, group, page = [150, 0, 65, 1], 2, 3, 24
    pages, table = spread(jot, 31, lens, nkv, page, hd, dtype, width=9, joined=True, layers=3)
    wide = normal(5, (4, T, nkv * group + 4, hd), dtype)
    q = wide[:, :, 2:2 + nkv * group]
    room = torch.full((T, 4, nkv * group + 1, hd), 7.0, dtype=dtype, device="cuda")
    out = room.transpose(0, 1)[:, :, :nkv * group]
    first, _ = check_attention(jot, q, pages, table, lens, layer=1, out=out)
    assert (room[:, :, -1] == 7.0).all()
    first = first.clone()
    for b, n in enumerate(lens):
        if n % page:
            p = int(table[b, n // page])
            pages.k[1, p, :, n % page:] = math.nan
            pages.v[1, p, :, n % page:] = math.inf
    used = set(table[table >= 0].tolist())
    for p in range(pages.n_pages):
        if p not in used:
            pages.v[1, p] = math.nan
    pages.v[0], pages.k[2] = math.nan, math.nan
    table[2, 4:] = 2 ** 30
    second, _ = check_attention(jot, q, pages, table, lens, layer=1, out=torch.full_like(first, 7.0))
    assert torch.equal(first, second)


def test_paged_attention_large_scores_and_scale(jot):
    """Scores of some hundreds (maxima that rise from tile to tile, probabilities that underflow) and another scale."""
    lens = [700, 64]
    for T in (1, 32, 80):
        pages, table = spread(jot, 41, lens, 2, 16, 64, BF16)
        q = normal(6, (2, T, 4, 64), BF16, 8.0)
        check_attention(jot, q, pages, table, lens, scale=1.0)
        check_attention(jot, q, pages, table, lens, scale=-0.01)
        pages.k[:] = 0                                      # all scores alike: the mean of the values
        check_attention(jot, q, pages, table, lens)


def test_paged_attention_infinite_and_nan_scores_reach_their_rows_only(jot):
    lens = [130, 130]
    pages, table = spread(jot, 43, lens, 1, 16, 64, BF16)
    q = normal(7, (2, 3, 2, 64), BF16)
    q[0, 1, 0] = math.nan
    out = jot.paged_attention(q, pages, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    bad = torch.zeros(2, 3, 2, dtype=torch.bool, device="cuda")
    bad[0, 1, 0] = True
    assert torch.equal(out.isnan().all(-1), bad) and torch.equal(out.isnan().any(-1), bad)


def test_paged_attention_bad_pages_and_lengths_are_reported_and_read_nothing(jot):
    lens = [100, 40]
    pages, table = spread(jot, 45, lens, 2, 16, 64, BF16)
    q = normal(8, (2, 5, 4, 64), BF16)
    good = jot.paged_attention(q, pages, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    for bad in (-1, -7, pages.n_pages, 2 ** 31 - 1):
        t = table.clone()
        t[0, 2] = bad
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = jot.paged_attention(q, pages, t.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), status=status)
        assert int(status) == jot.STATUS_BAD_INDEX
        assert torch.equal(out[1], good[1]) and out.isfinite().all()
    # a length beyond the table's row counts up to its end
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    t = table[:, :3].cuda()
    out = jot.paged_attention(q, pages, t, torch.tensor([100, 40], dtype=torch.int32, device="cuda"), status=status)
    assert int(status) == jot.STATUS_BAD_INDEX
    want = jot.paged_attention(q, pages, t, torch.tensor([48, 40], dtype=torch.int32, device="cuda"))
    assert torch.equal(out, want)
    # without a status word the result is the same
    assert torch.equal(jot.paged_attention(q, pages, t, torch.tensor([100, 40], dtype=torch.int32, device="cuda")), want)


def test_paged_attention_empty_calls(jot):
    pages, table = spread(jot, 47, [10], 2, 16, 64, BF16)
    lens = torch.tensor([10], dtype=torch.int32, device="cuda")
    assert jot.paged_attention(normal(1, (1, 0, 4, 64), BF16), pages, table.cuda(), lens, workspace=torch.empty(0, dtype=torch.uint8, device="cuda")).numel() == 0
    assert jot.paged_attention(normal(1, (0, 2, 4, 64), BF16), pages, table[:0].cuda(), lens[:0]).numel() == 0
    out = jot.paged_attention(normal(1, (1, 2, 4, 64), BF16), pages, table[:, :0].cuda(), lens)     # a table without entries
    assert (out == 0).all()
    freq = jot.rope_frequencies(64, 1e4)
    none = normal(1, (0, 4, 64), BF16)
    assert jot.head_norm_rope(none, none, lens[:0], jot.Rope(freq))[0].shape == (0, 4, 64)
    jot.kv_write(pages, none[:, :2], none[:, :2], lens[:0])
    jot.kv_copy_pages(pages, [], [])


def test_calls_on_two_streams_with_a_workspace_each(jot):
    lens = [3000, 700, 5]
    pages, table = spread(jot, 51, lens, 4, 16, 128, BF16)
    table, dl = table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    qs = [normal(10 + i, (3, 1 + 20 * i, 28, 128), BF16) for i in range(2)]
    want = [jot.paged_attention(q, pages, table, dl) for q in qs]
    ws = [torch.empty(jot.paged_attention_workspace_bytes(q.shape[1], 28, 4, 128), dtype=torch.uint8, device="cuda") for q in qs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                outs[i].append(jot.paged_attention(qs[i], pages, table, dl, workspace=ws[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in outs[i])


def test_a_block_pass_put_together_and_replayed_as_a_graph(jot):
    """What a step does with a layer: projection, norm and rotation into the pages, attention over the pages, projection; twice
    eagerly and as a captured graph whose tokens, positions, slots, tables and lengths have changed since the capture."""
    B, T, nq, nkv, hd, page, d = 3, 8, 4, 2, 64, 16, 256
    wqkv, wo = normal(1, ((nq + 2 * nkv) * hd, d), BF16, 0.06), normal(2, (d, nq * hd), BF16, 0.06)
    gain = (1 + 0.1 * normal(3, (hd,), torch.float32)).to(BF16)
    rope = jot.Rope(jot.rope_frequencies(hd, 1e4))
    start = spread(jot, 61, [120] * B, nkv, page, hd, BF16, width=8)
    ws = torch.empty(jot.paged_attention_workspace_bytes(T, nq, nkv, hd), dtype=torch.uint8, device="cuda")

    def inputs(seed, firsts):
        """Rows T of each sequence at positions first ..; a first of None: the sequence idles."""
        x = normal(seed, (B * T, d), BF16)
        pos = torch.tensor([[-1] * T if f is None else list(range(f, f + T)) for f in firsts], dtype=torch.int32)
        lens = torch.tensor([-1 if f is None else f + T for f in firsts], dtype=torch.int32)
        slots = torch.where(pos < 0, -1, torch.gather(start[1].long(), 1, pos.clamp(min=0).long() // page).int() * page + pos % page).int()
        return [x, pos.flatten().cuda(), slots.flatten().cuda(), lens.cuda()]

    def step(pages, x, pos, slots, lens, table, qkv, att):
        # the projection's entry point reads its status back, which a capture does not allow: the library call itself
        lib, st = jot._lib(), torch.cuda.current_stream().cuda_stream
        assert lib.jot_gemm_bf16(x.data_ptr(), wqkv.data_ptr(), None, qkv.data_ptr(), B * T, qkv.shape[1], d, None, 0, None, st) == 0
        q, k, v = qkv.view(B * T, nq + 2 * nkv, hd).split([nq, nkv, nkv], 1)
        jot.head_norm_rope(q, k, pos, rope, gain, gain, q_out=q, v=v, pages=pages, slots=slots)
        jot.paged_attention(q.unflatten(0, (B, T)), pages, table, lens, out=att, workspace=ws)
        y = torch.empty(B * T, d, dtype=BF16, device="cuda")
        assert lib.jot_gemm_bf16(att.data_ptr(), wo.data_ptr(), x.data_ptr(), y.data_ptr(), B * T, d, nq * hd, None, 0, None, st) == 0
        return y

    def eager(args, table):
        pages = jot.KVPages(start[0].k.clone(), start[0].v.clone())
        att = torch.zeros(B, T, nq, hd, dtype=BF16, device="cuda")
        return step(pages, *args, table, torch.empty(B * T, (nq + 2 * nkv) * hd, dtype=BF16, device="cuda"), att), pages

    first, second = inputs(70, [100, 3, None]), inputs(71, [0, None, 112])
    table = start[1].cuda()
    # the eager result, against the definitions
    y, pages = eager(first, table)
    x64 = first[0].double().cpu()
    qkv = (x64 @ wqkv.double().cpu().T).to(BF16).view(B * T, nq + 2 * nkv, hd)
    got_k = pages.k[0]
    want_k, size = rope_wanted(qkv[:, nq:nq + nkv], first[1], rope.inv_freq, False, 1.0, gain, 1e-6)
    for r in range(2 * T):
        at = got_k[first[2][r] // page, :, first[2][r] % page].double().cpu()
        # the projection is rounded to bf16 on either side of a tie: one step of it, and the rotation's own rounding
        assert ((at - want_k[r]).abs() <= 2.0 ** -7 * size[r] * 2 ** 0.5 + 2.0 ** -8 * want_k[r].abs() + 1e-3).all()
    q = jot.head_norm_rope(qkv[:, :nq].cuda().contiguous(), None, first[1], rope, gain)[0]
    check_attention(jot, q.view(B, T, nq, hd), pages, start[1], first[3].tolist())
    # captured once, replayed with other contents
    static = [t.clone() for t in first]
    g_pages = jot.KVPages(start[0].k.clone(), start[0].v.clone())
    g_qkv, g_att = torch.empty(B * T, (nq + 2 * nkv) * hd, dtype=BF16, device="cuda"), torch.zeros(B, T, nq, hd, dtype=BF16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g_y = step(g_pages, *static, table, g_qkv, g_att)
    for args in (second, first):
        g_pages.k.copy_(start[0].k), g_pages.v.copy_(start[0].v), g_att.zero_()
        for a, b in zip(static, args):
            a.copy_(b)
        graph.replay()
        want_y, want_pages = eager(args, table)
        assert torch.equal(g_y, want_y) and torch.equal(g_pages.k, want_pages.k) and torch.equal(g_pages.v, want_pages.v)


def test_refusals_on_the_device(jot):
    """What the binding lets through and the library refuses, before anything is launched."""
    pages, table = spread(jot, 81, [40], 2, 16, 64, BF16)
    table, lens, q = table.cuda(), torch.tensor([40], dtype=torch.int32, device="cuda"), normal(1, (1, 2, 4, 64), BF16)
    n0 = jot.launch_count()

    def refused(status, fn):
        with pytest.raises(jot.JotError) as e:
            fn()
        assert e.value.status == status

    small = torch.empty(64, dtype=torch.uint8, device="cuda")
    refused(-3, lambda: jot.paged_attention(q, pages, table, lens, workspace=small))
    refused(-2, lambda: jot.paged_attention(normal(1, (1, 2, 3, 64), BF16), pages, table, lens, workspace=small))
    refused(-1, lambda: jot.paged_attention(q, pages, table, lens, layer=1))
    refused(-1, lambda: jot.paged_attention(q, pages, table, lens, scale=math.nan))
    refused(-1, lambda: jot.paged_attention(normal(1, (1, 2, 4, 65), BF16)[..., 1:], pages, table, lens))     # odd strides
    wide = jot.KVPages(torch.zeros(1, 2, 1, 8, 256, dtype=BF16, device="cuda"), torch.zeros(1, 2, 1, 8, 256, dtype=BF16, device="cuda"))
    refused(-2, lambda: jot.paged_attention(normal(1, (1, 2, 4, 256), BF16), wide, table, lens, workspace=small))
    rows = torch.arange(3, dtype=torch.int32, device="cuda")
    x = normal(1, (3, 4, 64), BF16)
    refused(-2, lambda: jot.head_norm_rope(x, None, rows, jot.Rope(jot.rope_frequencies(24, 1e4))))
    refused(-1, lambda: jot.head_norm_rope(x, None, rows, jot.Rope(jot.rope_frequencies(80, 1e4))))
    refused(-1, lambda: jot.kv_write(pages, x[:, :2], x[:, 2:], rows, layer=-1))
    for src, dst in (([0], [pages.n_pages]), ([-1], [0]), ([0, 1], [2, 2]), ([0, 1], [1, 2]), ([0], [0])):
        refused(-1, lambda: jot.kv_copy_pages(pages, src, dst))
    for pages_bad in ([2 ** 32], [-2 ** 31 - 1]):
        with pytest.raises(OverflowError):
            jot.kv_copy_pages(pages, pages_bad, [1])
    assert jot.launch_count() == n0
    for bad in (lambda: jot.paged_attention(q.half(), pages, table, lens), lambda: jot.paged_attention(q, pages, table.long(), lens),
                lambda: jot.paged_attention(q, pages, table, lens.cpu()), lambda: jot.head_norm_rope(x.float(), None, rows, jot.Rope(jot.rope_frequencies(64, 1e4))),
                lambda: jot.kv_write(pages, x[:, :2].half(), x[:, 2:], rows), lambda: jot.KVPages(pages.k, pages.v.half()),
                lambda: jot.KVPages(pages.k.transpose(2, 3), pages.v.transpose(2, 3))):
        with pytest.raises(TypeError):
            bad()
    assert jot.launch_count() == n0
