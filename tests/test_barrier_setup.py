"""Barriers in shared memory that asynchronous copies or other blocks signal are set up with the fences that make the set-up
visible to them (host only, read from the sources: what is missing there shows on no GPU until it does)."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2312_00752_b200", "csrc")


def _sources():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))):
        yield os.path.basename(path), re.sub(r"//[^\n]*", "", open(path).read())


def test_every_barrier_set_up_is_followed_by_its_fences():
    seen = 0
    for name, text in _sources():
        for m in re.finditer(r"mbarrier\.init", text):
            end = text.index("\n}", m.end())                    # of the function that it is in
            following = text[m.end():end]
            sync = re.search(r"__syncthreads|cluster_sync|barrier\.cluster", following)
            before = following[:sync.start()] if sync else following
            assert "fence.mbarrier_init.release.cluster" in before, name
            assert "fence.proxy.async.shared::cta" in before, name
            seen += 1
    assert seen > 0


def test_barriers_are_signalled_only_where_that_function_sets_them_up():
    # (a kernel's own file calls it; the helpers of a header serve the files that include it)
    for name, text in _sources():
        if name.endswith(".cu") and re.search(r"barrier_expect\(|\bexpect\(|expect_tx", text):
            assert re.search(r"if \(threadIdx\.x == 0\) set_up_barriers\(\w+, \w+\);\s*(__syncthreads|cluster_sync)\(\);", text), name
