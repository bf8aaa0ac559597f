"""Source checks of what the update's kernels do where a bounded wait runs out (no GPU: no wait does)."""
import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2106_06998_b200", "csrc", "update", "newton_schulz.cu")


def _function(name):
    code = re.sub(r"//[^\n]*", "", open(SOURCE).read())
    return code.split(name + "(", 1)[1].split("\n}\n")[0]


def test_every_wait_of_the_small_matrices_kernel_is_looked_at():
    """After each of the three: nothing of the sums is read and no operand written by a warp whose wait ran out, the block agrees on it at the next barrier, and no
    result is written behind it.  The last wait of such a warp, again with a limit, is the one before the tensor memory is given back."""
    body = _function("void small_steps")
    waits = [m.start() for m in re.finditer(r"\bwait\(\)", body)]
    assert len(waits) == 4 and len(re.findall(r"\bok = wait\(\);", body)) == 3 and body.rstrip().endswith("if (!ok) wait();")
    for at, following in zip(waits[:3], waits[1:]):
        part = body[at:following]
        guarded = part.index("lost = __syncthreads_or(!ok);")
        assert "__syncthreads()" not in part[:guarded]
        for use in re.finditer(r"small_sums<|st_shared_v4\(|st\.shared\.v4", part[:guarded]):
            assert re.search(r"if \(ok\)|; ok && b < here;", part[:use.start()])
    assert len(re.findall(r"!lost; [cb]0 \+= ", body)) == 2 and "if (last && !lost) {" in body and body.count("small_write(") == 1
    assert body.index("if (last && !lost) {") < body.index("small_write(")


def test_the_ctas_of_a_cluster_end_together():
    """The word that says so is written before the first of a step's two cluster barriers and read between them, by every thread."""
    body = _function("void small_steps")
    syncs = [m.start() for m in re.finditer(r"cluster_sync\(\);", body)]
    assert len(syncs) == 2
    assert body.index("st_cluster_u32(smem_u32(gone)") < syncs[0] < body.index("reinterpret_cast<volatile uint32_t*>(gone) != 0) break;") < syncs[1]
    assert "if (lost) break;" in body[syncs[1]:] and "if (lost && p.cs == 1) break;" in body       # (a CTA by itself: at once)
    kernel = _function("void __launch_bounds__(SMALL_THREADS, 1) ns_small_kernel")
    assert kernel.index("gone = 0;") < kernel.index("cluster_sync();") and kernel.count("&gone)") == 2


def test_a_shared_tile_without_all_its_sums_is_not_written():
    kernel = _function("ns_product_kernel")
    told, read = kernel.index("if (!ok && shared && lane < 2 * p.cs) st_cluster_u32(smem_u32(&lost)"), kernel.index("reinterpret_cast<volatile uint32_t*>(&lost) == 0")
    syncs = [m.start() for m in re.finditer(r"\bcluster_sync\(\);", kernel)]
    assert kernel.index("lost = 0;") < syncs[0] < told < syncs[-1] < read < kernel.index("ns_emit<MODE, 1>(")
