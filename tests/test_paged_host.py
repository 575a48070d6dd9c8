"""The host side of the paged cache: what the library refuses before it touches a device, the frequencies of a rotation, and the pool
that says which sequence has which page (against a model of the cache's contents)."""
import ctypes as C
import math
import random

import pytest
import torch

from paper_2602_11133_b200 import build as jot_build
from paper_2602_11133_b200.kv_pages import OutOfPages, PagePool

ARG, SHAPE, WORKSPACE = -1, -2, -3
PTR = 4096                                  # an aligned address that nothing dereferences: every check below comes first


@pytest.fixture(scope="module")
def jot():
    jot_build.build()
    from paper_2602_11133_b200 import jot as binding
    binding._lib()
    return binding


def pages_struct(jot, **kw):
    d = dict(k=PTR, v=PTR, k_layer_stride=0, v_layer_stride=0, k_page_stride=4 * 16 * 64, v_page_stride=4 * 16 * 64, n_layers=1, n_pages=8, n_kv_heads=4,
             page_size=16, head_dim=64, dtype=0)
    d.update(kw)
    order = ("k", "v", "k_layer_stride", "v_layer_stride", "k_page_stride", "v_page_stride", "n_layers", "n_pages", "n_kv_heads", "page_size", "head_dim", "dtype")
    return jot._pack_pages(*(d[x] or 0 for x in order))


BAD_PAGES = [(dict(k=None), ARG), (dict(v=PTR + 8), ARG), (dict(n_pages=0), ARG), (dict(page_size=-1), ARG), (dict(dtype=2), ARG), (dict(head_dim=60), SHAPE),
             (dict(n_pages=2 ** 30), SHAPE), (dict(k_page_stride=4 * 16 * 64 - 8), ARG), (dict(v_page_stride=4 * 16 * 64 + 4), ARG),
             (dict(n_layers=2, k_layer_stride=12), ARG)]


@pytest.mark.parametrize("change,status", BAD_PAGES)
def test_pages_that_are_refused_everywhere(jot, change, status):
    lib, p = jot._lib(), pages_struct(jot, **change)
    assert lib.jot_kv_write(p, 0, 1, PTR, 256, 64, PTR, 256, 64, PTR, None, None) == status
    one = (C.c_int32 * 1)(0)
    assert lib.jot_kv_copy_pages(p, 1, one, (C.c_int32 * 1)(1), None) == status
    assert lib.jot_paged_attention(PTR, 256, 256, 64, PTR, 256, 256, 64, None, 1, 1, 4, p, 0, PTR, 4, 4, PTR, 1.0, PTR, 1 << 30, None, None) == status
    assert lib.jot_paged_attention(PTR, 256, 256, 64, PTR, 256, 256, 64, None, 1, 1, 4, None, 0, PTR, 4, 4, PTR, 1.0, PTR, 1 << 30, None, None) == ARG


def test_layers_out_of_range_are_refused(jot):
    lib, p = jot._lib(), pages_struct(jot)
    for layer in (-1, 1):
        assert lib.jot_kv_write(p, layer, 1, PTR, 256, 64, PTR, 256, 64, PTR, None, None) == ARG


def test_head_norm_rope_refusals(jot):
    lib = jot._lib()
    H = lambda n=4, src=PTR, out=PTR, row=256, head=64, gain=None: jot._pack_heads(src, row, head, out or 0, row, head, gain or 0, n)
    rope = lambda rotary=64, il=0, freq=PTR: jot._pack_rope(freq or 0, rotary, il, 1.0)

    def call(q=None, k=None, r=None, dtype=0, rows=2, hd=64, pos=PTR, v=None, pages=None, layer=0, slots=None):
        return lib.jot_head_norm_rope(q or H(), k, r or rope(), dtype, rows, hd, 1e-6, pos, v, pages, layer, slots, None, None)

    assert call(rows=0) == 0 and call(rows=0, pos=None) == 0
    assert call(rows=-1) == ARG and call(dtype=5) == ARG and call(pos=None) == ARG
    assert call(hd=4) == SHAPE and call(hd=264) == SHAPE and call(hd=68) == SHAPE
    assert call(r=rope(128)) == ARG and call(r=rope(64, freq=None)) == ARG
    assert call(r=rope(24)) == SHAPE and call(r=rope(4, 1)) == SHAPE
    assert call(q=H(0)) == ARG and call(q=H(src=PTR + 2)) == ARG and call(q=H(row=260)) == ARG and call(q=H(head=60)) == ARG and call(q=H(gain=PTR + 8)) == ARG
    assert call(q=H(out=None)) == ARG and call(k=H(out=None)) == ARG
    assert call(v=H()) == ARG                                            # values go to pages only
    p = pages_struct(jot)
    assert call(pages=p, k=H(), v=None, slots=PTR) == ARG and call(pages=p, k=None, v=H(), slots=PTR) == ARG and call(pages=p, k=H(), v=H()) == ARG
    assert call(pages=p, k=H(2), v=H(2), slots=PTR) == ARG and call(pages=p, k=H(), v=H(2), slots=PTR) == ARG and call(pages=p, k=H(), v=H(), slots=PTR, dtype=1) == ARG
    assert call(pages=p, k=H(), v=H(), slots=PTR, layer=1) == ARG


def test_counts_beyond_31_bits_are_refused(jot):
    # the kernels count rows and heads in 31 bits, up to the end of the last CTA's rows
    lib, p, most = jot._lib(), pages_struct(jot), 2 ** 31 - 1
    heads = lambda n: jot._pack_heads(PTR, 8, 8, PTR, 8, 8, 0, n)
    rope = jot._pack_rope(0, 0, 0, 1.0)
    assert lib.jot_head_norm_rope(heads(1), None, rope, 0, most, 8, 1e-6, PTR, None, None, 0, None, None, None) == SHAPE
    assert lib.jot_head_norm_rope(heads(most), None, rope, 0, 1, 8, 1e-6, PTR, None, None, 0, None, None, None) == SHAPE
    assert lib.jot_head_norm_rope(heads(1), heads(most), rope, 0, 1, 8, 1e-6, PTR, None, None, 0, None, None, None) == SHAPE
    assert lib.jot_kv_write(p, 0, most, PTR, 256, 64, PTR, 256, 64, PTR, None, None) == SHAPE


def test_copy_lists_that_hang_on_their_order_are_refused(jot):
    lib, p = jot._lib(), pages_struct(jot, n_pages=100)

    def copy(src, dst, n=None):
        return lib.jot_kv_copy_pages(p, len(src) if n is None else n, (C.c_int32 * max(1, len(src)))(*src), (C.c_int32 * max(1, len(dst)))(*dst), None)

    assert copy([], []) == 0 and copy([], [], -1) == ARG
    assert copy([100], [0]) == ARG and copy([0], [-1]) == ARG and copy([3], [3]) == ARG
    assert copy([0, 1], [2, 2]) == ARG and copy([0, 1], [1, 2]) == ARG and copy([0, 2], [1, 0]) == ARG
    many = list(range(45))                                               # the form for longer lists
    assert copy(many, many[:-1] + [99]) == ARG and copy(many, [50 + i for i in many[:-1]] + [50]) == ARG
    assert copy(many, [50 + i for i in many[:-1]] + [44]) == ARG


def test_paged_attention_refusals(jot):
    lib, p = jot._lib(), pages_struct(jot)

    def call(q=PTR, strides=(256, 256, 64), out=PTR, B=1, T=1, nq=4, pages=p, layer=0, table=PTR, stride=4, width=4, lens=PTR, scale=1.0, ws=PTR, nbytes=1 << 30):
        return lib.jot_paged_attention(q, *strides, out, *strides, None, B, T, nq, pages, layer, table, stride, width, lens, scale, ws, nbytes, None, None)

    assert call(B=0) == 0 and call(T=0) == 0
    assert call(B=-1) == ARG and call(T=-1) == ARG and call(nq=0) == ARG and call(width=-1) == ARG and call(stride=-1) == ARG
    assert call(q=None) == ARG and call(out=None) == ARG and call(lens=None) == ARG and call(table=None) == ARG and call(q=PTR + 2) == ARG
    assert call(strides=(256, 256, 63)) == ARG and call(T=2, strides=(256, 250, 64)) == ARG
    assert call(scale=math.inf) == ARG and call(scale=math.nan) == ARG
    assert call(nq=6) == SHAPE and call(pages=pages_struct(jot, head_dim=80, k_page_stride=4 * 16 * 80, v_page_stride=4 * 16 * 80)) == SHAPE
    assert call(width=2 ** 31 // 16) == SHAPE and call(B=2 ** 20, width=2 ** 20) == SHAPE          # more tiles of keys than the kernels count
    assert call(ws=None) == WORKSPACE and call(ws=PTR + 4) == WORKSPACE and call(nbytes=1000) == WORKSPACE
    assert [jot.paged_attention_workspace_bytes(*a) for a in ((0, 4, 4, 64), (1, 4, 3, 64), (1, 4, 4, 80), (-1, 4, 4, 64), (2 ** 31 - 1, 64, 1, 64))] == [0] * 5
    sizes = [jot.paged_attention_workspace_bytes(t, 4, 4, 128) for t in (1, 16, 17, 32, 64, 128, 129, 5000)]
    assert all(s > 0 for s in sizes) and sizes[0] == sizes[1] and sizes[2] == sizes[3] and sizes[6] == sizes[7]


def test_attaching_pages_refusals(jot):
    lib = jot._lib()
    assert lib.jot_attach_kv_pages(None, None, None, 0, 0, None, 0) == ARG
    cfg = jot.ModelConfig(2, 256, 4, 4, 64, 704, 4096, 4095, 10000.0, 1e-5)
    assert lib.jot_kv_pages_workspace_bytes(C.byref(cfg), 0, 96) == 0 and lib.jot_kv_pages_workspace_bytes(C.byref(cfg), 1, 0) == 0
    n1, n2 = (lib.jot_kv_pages_workspace_bytes(C.byref(cfg), b, 96) for b in (1, 2))
    assert 0 < n1 < n2


def test_rope_frequencies(jot):
    f = jot.rope_frequencies(64, 10000.0, device="cpu").double()
    want = 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)
    assert f.dtype == torch.float64 and ((f - want).abs() <= 2.0 ** -24 * want).all()
    assert torch.equal(jot.rope_frequencies(64, 10000.0, 4.0, device="cpu"), (want / 4).float())
    by_turns = jot.rope_frequencies(64, 10000.0, 4.0, 8192, 1.0, 4.0, device="cpu").double()
    turns = 8192 * want / (2 * math.pi)
    assert torch.equal(by_turns[turns >= 4].float(), want[turns >= 4].float())
    assert torch.equal(by_turns[turns <= 1].float(), (want[turns <= 1] / 4).float())
    between = (turns > 1) & (turns < 4)
    assert between.any() and ((by_turns < want) & (by_turns > want / 4))[between].all()
    assert (by_turns[1:] < by_turns[:-1]).all()
    for bad in ((0, 1e4), (63, 1e4), (64, 0.0), (64, 1e4, 0.0), (64, 1e4, 2.0, 8192, 4.0, 4.0)):
        with pytest.raises(ValueError):
            jot.rope_frequencies(*bad, device="cpu")


# ---------------------------------------------------------------------------------------------- the pool
def check(pool, content, memory):
    """Every sequence reads what was written to it; pages add up."""
    users = {}
    for s, want in content.items():
        assert pool.length(s) == len(want)
        slots = pool.slots(s, range(len(want)))
        assert [memory[x] for x in slots] == want
        assert len(pool.pages(s)) == (len(want) + pool.page_size - 1) // pool.page_size
        for p in pool.pages(s):
            users[p] = users.get(p, 0) + 1
    assert pool.free_pages == pool.n_pages - len(users)


@pytest.mark.parametrize("page_size,seed", [(1, 0), (4, 1), (16, 2), (5, 3)])
def test_pool_against_a_model_of_the_contents(page_size, seed):
    rng, pool, content, memory, names = random.Random(seed), PagePool(40, page_size), {}, {}, 0

    def copy(pair):
        src, dst = pair
        assert len(src) == len(dst) and len(set(dst)) == len(dst) and not set(src) & set(dst)
        before = dict(memory)
        for a, b in zip(src, dst):
            for o in range(page_size):
                memory[b * page_size + o] = before.get(a * page_size + o)

    def write(s, lo, hi):
        copy(pool.own(s, lo, hi))
        for i, slot in zip(range(lo, hi), pool.slots(s, range(lo, hi))):
            content[s][i] = memory[slot] = rng.random()

    for _ in range(600):
        op = rng.choice(["add", "fork", "write", "resize", "free", "compact"])
        s = rng.choice(list(content)) if content else None
        try:
            if op == "add":
                n = rng.randint(0, 6 * page_size)
                pool.add(names, n)
                content[names] = [None] * n
                names += 1
                write(names - 1, 0, n)
            elif s is None:
                continue
            elif op == "fork":
                pool.fork(s, names)
                content[names] = list(content[s])
                names += 1
            elif op == "write":
                n = len(content[s])
                lo = rng.randint(0, n)
                write(s, lo, rng.randint(lo, n))
            elif op == "resize":
                n, old = rng.randint(0, 6 * page_size), len(content[s])
                pool.resize(s, n)
                content[s] = (content[s] + [None] * n)[:n]
                if n > old:
                    write(s, old, n)
            elif op == "free":
                pool.free(s)
                del content[s]
            else:
                copy(pool.compact())
                used = {p for x in content for p in pool.pages(x)}
                assert used == set(range(len(used)))
        except OutOfPages:
            # nothing changed, but a write after a resize or an add may be what did not fit: those positions hold nothing yet
            for x in content:
                content[x] = (content[x] + [None] * pool.length(x))[:pool.length(x)]
                for i, slot in enumerate(pool.slots(x, range(len(content[x])))):
                    if content[x][i] is None:
                        content[x][i] = memory.get(slot)
        check(pool, content, memory)


def test_pool_refusals():
    pool = PagePool(4, 16)
    pool.add("a", 33)
    assert pool.free_pages == 1 and pool.table(["a"], 5) == [[0, 1, 2, -1, -1]]
    with pytest.raises(OutOfPages):
        pool.add("b", 17)
    assert pool.free_pages == 1
    with pytest.raises(KeyError):
        pool.length("b")
    for bad in (lambda: pool.add("a", 1), lambda: pool.fork("a", "a"), lambda: pool.resize("a", -1), lambda: pool.own("a", 0, 34), lambda: pool.own("a", 5, 4),
                lambda: pool.slots("a", [33]), lambda: pool.slots("a", [-1]), lambda: pool.table(["a"], 2), lambda: pool.add("c", -1), lambda: PagePool(0, 1)):
        with pytest.raises(ValueError):
            bad()
    pool.fork("a", "c")
    with pytest.raises(OutOfPages):
        pool.own("c", 0, 33)                # three pages wanted, one free: nothing has changed
    assert pool.pages("a") == pool.pages("c") and pool.own("c", 32, 33) == ([2], [3]) and pool.pages("c") == [0, 1, 3]
    pool.free("a")
    assert pool.free_pages == 1 and pool.own("c", 0, 33) == ([], [])
