"""The model's cache where it can go wrong: attached while a stream is busy, filled by a pass that failed, its status word."""
import pytest
import torch

from paper_2602_11133_b200 import inputs
from test_gpu_kv_pages import in_pages, jot  # noqa: F401 (jot: the fixture)
from test_gpu_kvcache import GEOMS

pytestmark = pytest.mark.gpu


def small(jot, B=2, P=40, G=56, name="gqa"):
    g = GEOMS[name]
    model = jot.Model(g, inputs.weights_to(inputs.model_weights(g, seed=0), "cuda"), B, P + G)
    canvas = inputs.partially_masked_canvas(1, B, P, G, g.vocab, g.mask_id, 0.8)
    canvas[:, P:P + 16] = g.mask_id
    return g, model, canvas.cuda(), P, P + 16


def control(model):
    """The model's status word."""
    at = -model.workspace.data_ptr() % 1024
    return model.workspace[at:at + 4].view(torch.int32)


def refused(jot, status, fn):
    with pytest.raises(jot.JotError) as e:
        fn()
    assert e.value.status == status


@pytest.mark.parametrize("word,status", [(1, -5), (2, -5), (3, -5), (4, -5), (7, -5), (8, -5), (5, -1), (6, -1)])
def test_what_the_status_words_of_the_kernels_mean(jot, word, status):
    _, model, _, _, _ = small(jot)
    control(model).fill_(word)
    refused(jot, status, model.read_status)
    # what the caller can mend is taken off the record, an expired wait stays
    assert int(control(model)) == (0 if status == -1 else word)
    model.close()


def test_a_bad_page_does_not_take_an_expired_wait_off_the_record(jot):
    g, model, canvas, lo, hi = small(jot)
    _, table = in_pages(jot, model, g, 2, canvas.shape[1], 16)
    model.denoise_step_cached(canvas, lo, hi, refresh=True)
    control(model).fill_(3)
    table[1, 0] = 10 ** 6
    refused(jot, -5, lambda: model.denoise_step_cached(canvas, lo, hi, refresh=False))
    model.close()


def test_a_bad_page_of_an_earlier_pass_is_reported_once_by_generate(jot):
    g, model, canvas, lo, hi = small(jot)
    _, table = in_pages(jot, model, g, 2, canvas.shape[1], 16)
    prompt = inputs.prompt(3, 2, 40, g.vocab, g.mask_id).cuda()
    model.set_sync(False)
    table[1, 0] = 10 ** 6
    model.denoise_step_cached(canvas, lo, hi, refresh=True)
    refused(jot, -1, lambda: model.generate(prompt, 56, 14, jot.Params(), block_len=28))
    model.generate(prompt, 56, 14, jot.Params(), block_len=28)
    model.close()


@pytest.mark.parametrize("paged", [True, False])
@pytest.mark.parametrize("sync", [True, False])
def test_a_refresh_that_failed_leaves_no_canvas(jot, paged, sync):
    """Blocks are attended over what a refresh left; one that was told of a bad page or a bad token left a mixture."""
    g, model, canvas, lo, hi = small(jot)
    if paged:
        _, table = in_pages(jot, model, g, 2, canvas.shape[1], 16)
    else:
        model.attach_kv_cache()
    block = lambda: model.denoise_step_cached(canvas, lo, hi, refresh=False)
    model.set_sync(sync)

    def failing_refresh():
        bad = canvas.clone()
        if paged:
            good = table.clone()
            table[1, 1] = 10 ** 6
        else:
            bad[0, 0] = g.vocab + 3
        if sync:
            refused(jot, -1, lambda: model.denoise_step_cached(bad, lo, hi, refresh=True))
        else:
            model.denoise_step_cached(bad, lo, hi, refresh=True)
            refused(jot, -1, model.read_status)
        if paged:
            table.copy_(good)

    failing_refresh()
    refused(jot, -1, block)
    model.denoise_step_cached(canvas, lo, hi, refresh=True)
    want = block().sumexp.clone()
    failing_refresh()
    refused(jot, -1, block)                                        # (the refresh before the failing one was of the same shape)
    model.denoise_step_cached(canvas, lo, hi, refresh=True)
    assert torch.equal(block().sumexp, want)
    # calls that are refused before anything is enqueued touch no cache
    with pytest.raises(jot.JotError):
        model.denoise_step_cached(canvas, lo, canvas.shape[1] + 1, refresh=True)
    assert torch.equal(block().sumexp, want)
    # a block that fails leaves the rest of the canvas alone: it can be run again
    bad = canvas.clone()
    bad[0, lo] = g.vocab + 3
    if sync:
        refused(jot, -1, lambda: model.denoise_step_cached(bad, lo, hi, refresh=False))
    else:
        model.read_status()
        model.denoise_step_cached(bad, lo, hi, refresh=False)
        refused(jot, -1, model.read_status)
    assert torch.equal(block().sumexp, want)
    model.set_sync(True)
    model.read_status()
    model.close()


def test_a_later_failure_is_not_the_refresh_s(jot):
    """Without a read in between, the refresh's own outcome tells whether there is a canvas, not what a later step met."""
    g, model, canvas, lo, hi = small(jot)
    _, table = in_pages(jot, model, g, 2, canvas.shape[1], 16)
    block = lambda c=canvas: model.denoise_step_cached(c, lo, hi, refresh=False)
    model.denoise_step_cached(canvas, lo, hi, refresh=True)
    want = block().sumexp.clone()
    bad = canvas.clone()
    bad[0, lo] = g.vocab + 3
    model.set_sync(False)
    for later in (lambda: block(bad), lambda: model.denoise_step(bad, lo, hi)):
        model.denoise_step_cached(canvas, lo, hi, refresh=True)
        later()
        refused(jot, -1, model.read_status)
        assert torch.equal(block().sumexp, want)
        model.read_status()
    # and the other way about: the steps behind a refresh that failed change nothing about it
    good = table.clone()
    table[1, 1] = 10 ** 6
    model.denoise_step_cached(canvas, lo, hi, refresh=True)
    table.copy_(good)
    block()
    refused(jot, -1, model.read_status)
    refused(jot, -1, block)
    model.close()


def test_a_generation_that_failed_leaves_no_canvas(jot):
    g, model, canvas, lo, hi = small(jot)
    _, table = in_pages(jot, model, g, 2, canvas.shape[1], 16)
    good = table.clone()
    prompt = inputs.prompt(3, 2, 40, g.vocab, g.mask_id).cuda()
    model.denoise_step_cached(canvas, lo, hi, refresh=True)
    table[1, 1] = -1
    refused(jot, -1, lambda: model.generate(prompt, 56, 14, jot.Params(), block_len=28, kv_cache=True))
    table.copy_(good)
    refused(jot, -1, lambda: model.denoise_step_cached(canvas, lo, hi, refresh=False))
    model.close()


def busy_block(nbytes):
    """On the current stream: a block of memory that a queued kernel will still write when the block is already free again."""
    block = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    torch.cuda._sleep(400_000_000)                                 # some 0.2 s
    block.fill_(0x55)
    return block.data_ptr()


def test_pages_attached_on_a_busy_stream(jot):
    """The workspace of attached pages may be memory that kernels queued on the stream have yet to write."""
    import ctypes as C
    g, model, canvas, lo, hi = small(jot)
    pages, table = in_pages(jot, model, g, 2, canvas.shape[1], 16)
    n = g.head_dim // 2
    want = model.kv_cache[2][:4 * n].view(torch.float32).clone()
    nbytes = jot._lib().jot_kv_pages_workspace_bytes(C.byref(model.cfg), 2, canvas.shape[1])
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        at = busy_block(nbytes)
        model.attach_kv_pages(pages, table)
        assert model.kv_cache[2].data_ptr() == at                  # the block, or this test shows nothing
        torch.cuda.synchronize()
        assert torch.equal(model.kv_cache[2][:4 * n].view(torch.float32), want)
    model.close()


def test_a_model_made_on_a_busy_stream(jot):
    g, model, canvas, lo, hi = small(jot)
    want = model.denoise_step(canvas, lo, hi).sumexp.clone()
    nbytes, w = model.workspace.numel(), model.weights
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        at = busy_block(nbytes)
        other = jot.Model(g, w, 2, canvas.shape[1])
        assert other.workspace.data_ptr() == at
        torch.cuda.synchronize()
        assert int(control(other)) == 0                            # (before any kernel works with what the model holds)
        assert torch.equal(other.denoise_step(canvas, lo, hi).sumexp, want)
    model.close(), other.close()
