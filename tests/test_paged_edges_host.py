"""Edges of the paged operators that need no device: status words, descriptors of cut items, arguments, the pool's checks."""
import glob
import os
import re
import subprocess

import pytest

from paper_2602_11133_b200 import build as jot_build
from paper_2602_11133_b200.kv_pages import PagePool

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_11133_b200", "csrc")


def sources():
    return {os.path.basename(p): open(p).read() for p in glob.glob(os.path.join(CSRC, "*.cu*"))}


def test_no_kernel_reports_an_expired_wait_as_bad_input():
    """The words of the caller's input (a token, an index) are answered as an argument error and taken off the record: a wait that expired
    must not look like one."""
    text = "\n".join(sources().values())
    of_input = {int(v) for v in re.findall(r"constexpr int32_t kStatusBad\w+ = (\d+);", text)}
    waits = [int(v) for v in re.findall(r"abort_flag && \w+\.status\) atomicExch\(\w+\.status, (\d+)\);", text)]
    assert len(of_input) == 2 and len(waits) >= 8
    assert not of_input & set(waits)


@pytest.fixture(scope="module")
def jot():
    jot_build.build()
    from paper_2602_11133_b200 import jot as binding
    binding._lib()
    return binding


def test_scales_whose_exponents_overflow_are_refused(jot):
    """Scores are scaled by scale * log2(e): a finite scale can make it infinite, and zero times it is no number."""
    lib = jot._lib()
    at = 4096                                  # an aligned address that nothing dereferences: the check comes first
    pages = jot._pack_pages(at, at, 0, 0, 4 * 16 * 64, 4 * 16 * 64, 1, 8, 4, 16, 64, 0)

    def call(scale):                           # without a workspace, which is looked at behind the scale
        return lib.jot_paged_attention(at, 256, 256, 64, at, 256, 256, 64, None, 1, 1, 4, pages, 0, at, 4, 4, at, scale, None, 0, None, None)

    assert [call(s) for s in (3e38, -3e38, 2.5e38)] == [-1] * 3
    assert [call(s) for s in (0.0, -0.0, 1e-45, 0.125, -0.125, 2.3e38)] == [-3] * 6


JOIN_CHECK = r"""
#include <climits>
#include <cstdio>
#include "paged_attention.cuh"
using namespace jot;
static unsigned long long seed = 88172645463325252ull;
static int any() { seed ^= seed << 13; seed ^= seed >> 7; seed ^= seed << 17; return (int)(seed >> 16); }
static int edge(int n) {                       // numbers around 0, n and the ends of the range, and any others
    const int at[] = {0, 1, -1, n - 1, n, n + 1, INT_MAX, INT_MIN, any(), any() % (2 * n + 1)};
    return at[(unsigned)any() % 10];
}
int main() {
    long taken = 0;
    for (int i = 0; i < 4000000; ++i) {        // whatever a workspace holds, a CTA reads parts within it and answers an item of its own
        const int shares = 1 + (unsigned)any() % 448, per_b = 1 + (unsigned)any() % 300, cta = (unsigned)any() % shares;
        const int4 d = make_int4(edge(shares), edge(shares), edge(shares), edge(shares));
        PagedJoin j;
        if (!paged_join_of(d, true, cta, per_b, shares, j)) continue;
        ++taken;
        if (j.b != cta / per_b || j.item != cta % per_b) return printf("item\n"), 1;
        if (j.share < 0 || j.parts < 1 || (long)j.share * 2 + 1 >= 2L * shares || ((long)j.share + j.parts - 1) * 2 >= 2L * shares) return printf("parts\n"), 1;
    }
    for (int ctas = 1; ctas < 450; ctas += 7)  // descriptors as they are written are all taken: an item of `n` tiles from tile `t` of a line on
        for (int total = ctas; total < 3000; total += 61)
            for (int t = 0; t < total; t += 13)
                for (int n : {1, 2, 30, 1000}) {
                    if (t + n > total) continue;
                    const int first = paged_owner(total, ctas, t), last = paged_owner(total, ctas, t + n - 1);
                    if (paged_share(total, ctas, first) > t || paged_share(total, ctas, first + 1) <= t) return printf("owner\n"), 1;
                    PagedJoin j;
                    if (last > first && !paged_join_of(make_int4(3, 5, last - first + 1, first), false, 9, 7, ctas, j)) return printf("refused\n"), 1;
                    if (last > first && (j.b != 3 || j.item != 5)) return printf("item by share\n"), 1;
                }
    printf("taken %ld\n", taken);
    return taken > 100000 ? 0 : 1;
}
"""


def test_descriptors_that_nobody_wrote_lead_nowhere(tmp_path):
    """A CTA that gives up on a wait leaves without describing its items, and the second kernel is on its way already: what stands in the
    workspace then must not become an address.  The kernel's own decision, compiled for the host."""
    (tmp_path / "join.cu").write_text(JOIN_CHECK)
    subprocess.run([jot_build._nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-O1", "-I", CSRC, "-o", str(tmp_path / "join"),
                    str(tmp_path / "join.cu")], check=True, capture_output=True, text=True)
    done = subprocess.run([str(tmp_path / "join")], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout
    # and the second kernel asks it before anything else of the descriptor is used
    kernel = sources()["paged_attention.cuh"].split("paged_join_kernel(")[1]
    assert kernel.count("a.desc[") == 1 and "if (!paged_join_of(a.desc[blockIdx.x], a.by_item, blockIdx.x, a.nkv * RT, shares, d)) return;" in kernel


def test_no_cta_leaves_with_copies_or_products_under_way():
    """A role that is through with its work cannot know that another one gives up after it: the copies it has sent are waited for, and the
    products it has issued, whether or not it has given up itself (what would happen otherwise cannot be tried out)."""
    text = sources()["paged_attention_umma.cuh"]
    producers = text.split("// ================================ producers")[1].split("// ================================ products")[0]
    drain = producers.split("for (int i = 0; i < RING; ++i) {")[1].split("\n            }")[0]
    assert "mbar_wait(&k_full[st], (nk - 1) & 1, &drain_flag)" in drain and "mbar_wait(&v_full[st], (nv - 1) & 1, &drain_flag)" in drain
    end = text.split("// ================================ products")[1].split("// ================================ softmax")[0].split("tails += has_tail;")[1]
    assert "if (ok) ok = wait_all(&v_empty[" in end and "if (!ok) {" in end and "umma_commit(&drain[s]);" in end and "mbar_wait(&drain[s], 0, &drain_flag);" in end


def test_lengths_that_are_no_integers_change_nothing_in_a_pool():
    pool = PagePool(4, 16)
    for call in (lambda: pool.add("a", 17.0), lambda: pool.add("a", "17"), lambda: pool.add("a", None)):
        with pytest.raises(TypeError):
            call()
        with pytest.raises(KeyError):
            pool.length("a")
    pool.add("a", 17)                          # the name is free
    with pytest.raises(TypeError):
        pool.resize("a", 16.5)                 # as many pages as before: it would have become a length
    assert pool.length("a") == 17 and pool.free_pages == 2
    with pytest.raises(TypeError):
        PagePool(4, 2.5)
