"""The block-wise KV cache in pages: the cached step against the CPU oracle and against the contiguous cache, Algorithm 1 over pages,
and pages that are forked, owned and moved between the steps of a run."""
import numpy as np
import pytest
import torch

from helpers import REL_TOL, compare_stats, oracle_stats_for_rows
from oracle import model_oracle as mo
from paper_2602_11133_b200 import inputs
from paper_2602_11133_b200.kv_pages import PagePool
from test_gpu_kvcache import GEOMS, fill_some

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def jot():
    from paper_2602_11133_b200 import jot as binding
    binding._lib()
    return binding


def in_pages(jot, model, g, B, L, page, seed=0, spare=5):
    """Attaches a pool whose sequences' pages lie in no order; returns (pages, table)."""
    each = (L + page - 1) // page
    ids = torch.randperm(B * each + spare, generator=torch.Generator().manual_seed(seed))
    table = ids[:B * each].view(B, each).int().cuda()
    pages = jot.KVPages.empty(len(model.weights["layers"]), B * each + spare, g.n_kv_heads, page, g.head_dim)
    pages.k.fill_(float("nan")), pages.v.fill_(float("nan"))       # whatever lies behind a canvas must not matter
    model.attach_kv_pages(pages, table)
    return pages, table


@pytest.mark.parametrize("name,B,P,G,lo,hi,page", [
    ("tiny", 1, 32, 64, 32, 64, 16),
    ("tiny", 2, 60, 140, 96, 112, 24),
    ("gqa", 3, 17, 120, 41, 65, 7),
    ("hd128", 2, 128, 256, 256, 384, 64),
    ("hd128", 1, 64, 320, 64, 224, 128),
])
def test_paged_cached_step_matches_oracle(jot, name, B, P, G, lo, hi, page):
    g = GEOMS[name]
    w_cpu = inputs.model_weights(g, seed=0)
    w_gpu = inputs.weights_to(w_cpu, "cuda")
    L = P + G
    canvas0 = inputs.partially_masked_canvas(1, B, P, G, g.vocab, g.mask_id, 0.8)
    canvas0[:, lo:hi] = g.mask_id
    canvas1 = fill_some(canvas0, g, lo, hi, seed=7)
    model = jot.Model(g, w_gpu, B, L)
    in_pages(jot, model, g, B, L, page)
    cache = []
    h0 = mo.hidden_states(g, w_cpu, canvas0, cache_out=cache)
    h1 = mo.hidden_states_cached(g, w_cpu, canvas1, cache, lo, hi)
    for canvas, refresh, h, first in ((canvas0, True, h0, 0), (canvas1, False, h1, lo)):
        st = model.denoise_step_cached(canvas.cuda(), lo, hi, refresh=refresh)
        rows = [(b, i) for b in range(B) for i in range(lo, hi) if int(canvas[b, i]) == g.mask_id]
        logits = mo.lm_head_logits(torch.stack([h[b, i - first] for b, i in rows]), w_cpu["lm_head"])
        want = oracle_stats_for_rows(logits, g.mask_id)
        flat = torch.tensor([b * L + i for b, i in rows])
        pick = lambda t: t.cpu().view(-1)[flat].numpy()
        n, near = compare_stats(pick(st.top1), pick(st.top2), pick(st.sumexp), pick(st.argmax), want, rel=REL_TOL)
        print(f"{name} [{lo},{hi}) refresh {refresh}: {n} rows, {near} near ties")
        assert near <= max(2, n // 20)
        untouched = torch.ones(B * L, dtype=torch.bool)
        untouched[flat] = False
        assert (st.sumexp.cpu().view(-1)[untouched] == 1.0).all()
    model.close()


def test_generate_over_pages_gives_the_contiguous_cache_s_tokens(jot):
    """With the planted bump every decision is far from its threshold, so the two caches' rounding differences change none."""
    g, B, P, G = GEOMS["gqa"], 3, 40, 96
    w = inputs.weights_to(inputs.model_weights(g, seed=0), "cuda")
    prompt = inputs.prompt(3, B, P, g.vocab, g.mask_id).cuda()
    ids, val = inputs.logit_bump(4, B, P + G, g.vocab, g.mask_id)
    val = (val + 20.0).cuda()
    got = []
    for paged in (False, True):
        model = jot.Model(g, w, B, P + G)
        if paged:
            in_pages(jot, model, g, B, P + G, 24)
        else:
            model.attach_kv_cache()
        out, used, passes = model.generate(prompt, G, 48, jot.Params(30.0, 1.0, 0.5, 8), block_len=32, bump_id=ids.cuda(), bump_val=val, kv_cache=True)
        got.append((out.cpu(), used, passes))
        model.close()
    assert torch.equal(got[0][0], got[1][0]) and got[0][1:] == got[1][1:]


def test_pages_move_and_fork_between_the_steps(jot):
    """The same block steps with the pages compacted between them, and for a fork of the first sequence whose shared pages are owned
    before they are written: the same bits, and the original's pages untouched by its fork."""
    g, P, G, page = GEOMS["hd128"], 70, 90, 16
    L, lo, hi = P + G, 80, 112
    w = inputs.weights_to(inputs.model_weights(g, seed=0), "cuda")
    canvas0 = inputs.partially_masked_canvas(1, 2, P, G, g.vocab, g.mask_id, 0.8)
    canvas0[:, lo:hi] = g.mask_id
    canvas1 = fill_some(canvas0, g, lo, hi, seed=3).cuda()
    canvas2 = fill_some(canvas1.cpu(), g, lo, hi, seed=4).cuda()
    pool = PagePool(64, page)
    pool.add("idle", 5 * page)                                     # in front of the others: what compaction moves them over
    pool.add("a", L)
    pool.add("b", L)
    pages = jot.KVPages.empty(2, 64, g.n_kv_heads, page, g.head_dim)
    table = torch.zeros(2, 12, dtype=torch.int32, device="cuda")
    model = jot.Model(g, w, 2, L)
    model.attach_kv_pages(pages, table)
    stats = lambda st: [t.clone() for t in (st.top1, st.top2, st.sumexp, st.argmax)]
    use = lambda *seqs: table.copy_(torch.tensor(pool.table(seqs, 12), dtype=torch.int32))

    use("a", "b")
    model.denoise_step_cached(canvas0.cuda(), lo, hi, refresh=True)
    k0, v0 = pages.k.clone(), pages.v.clone()
    plain = stats(model.denoise_step_cached(canvas1, lo, hi, refresh=False))
    # once more from the same refresh, with the pages moved to the pool's beginning first
    pages.k.copy_(k0), pages.v.copy_(v0)
    pool.free("idle")
    src, dst = pool.compact()
    assert len(src) == 5
    jot.kv_copy_pages(pages, src, dst)
    use("a", "b")
    moved = stats(model.denoise_step_cached(canvas1, lo, hi, refresh=False))
    assert all(torch.equal(x, y) for x, y in zip(plain, moved))
    # a fork of "a" takes another canvas' next step; "a" afterwards reads what it had
    mine = pool.slots("a", range(L))
    flat = lambda t: t.transpose(2, 3).reshape(2, -1, g.n_kv_heads, g.head_dim)[:, mine].clone()      # [layer, position, head, hd]
    before = flat(pages.k), flat(pages.v)
    pool.fork("a", "c")
    src, dst = pool.own("c", lo, hi)
    assert len(src) == 2                                           # positions 80..111: two whole pages of sixteen
    jot.kv_copy_pages(pages, src, dst)
    use("c", "b")
    forked = stats(model.denoise_step_cached(canvas2, lo, hi, refresh=False))
    assert torch.equal(flat(pages.k), before[0]) and torch.equal(flat(pages.v), before[1])
    use("a", "b")
    again = stats(model.denoise_step_cached(canvas2, lo, hi, refresh=False))
    assert all(torch.equal(x, y) for x, y in zip(forked, again))
    # a page outside the pool is an argument error, and the model goes on after it
    table[1, 3] = 64
    with pytest.raises(jot.JotError) as e:
        model.denoise_step_cached(canvas2, lo, hi, refresh=False)
    assert e.value.status == -1
    use("a", "b")
    model.denoise_step_cached(canvas2, lo, hi, refresh=False)
    # either cache takes the other's place
    model.attach_kv_cache()
    with pytest.raises(jot.JotError):
        model.denoise_step_cached(canvas2, lo, hi, refresh=False)
    model.detach_kv_cache()
    with pytest.raises(jot.JotError):
        model.denoise_step_cached(canvas2, lo, hi, refresh=True)
    model.close()


def test_attaching_pages_that_do_not_fit_is_refused(jot):
    g = GEOMS["gqa"]
    w = inputs.weights_to(inputs.model_weights(g, seed=0), "cuda")
    model = jot.Model(g, w, 2, 100)
    table = torch.zeros(2, 7, dtype=torch.int32, device="cuda")
    good = dict(n_layers=2, n_pages=20, n_kv_heads=2, page_size=16, head_dim=64)
    model.attach_kv_pages(jot.KVPages.empty(**good), table)
    for change, status in ((dict(n_layers=1), -1), (dict(n_kv_heads=4), -1), (dict(head_dim=128), -1), (dict(page_size=14), -2), (dict(dtype=torch.float16), -1)):
        with pytest.raises(jot.JotError) as e:
            model.attach_kv_pages(jot.KVPages.empty(**dict(good, **change)), table)
        assert e.value.status == status
    with pytest.raises(ValueError):
        model.attach_kv_pages(jot.KVPages.empty(**good), table[:1])
    with pytest.raises(TypeError):
        model.attach_kv_pages(jot.KVPages.empty(**good), table.long())
    model.close()
