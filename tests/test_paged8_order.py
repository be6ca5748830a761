"""Orders that the eviction's source has to keep and that no run can be relied on to show."""
import re

from test_source_order import REMOTE, START, kernel_body


def test_remote_shared_memory_after_a_cluster_barrier():
    body = kernel_body("paged8_evict.cu", "paged8_evict_kernel")
    remote = re.search(REMOTE, body).start()
    starts = [m for m in re.finditer(START, body[:remote])]
    assert starts, "no cluster barrier before the first access to another CTA's shared memory"
    # in the block of the loop over the passes that the access stands in, or around it: every CTA that gets there has passed it
    between = body[starts[-1].end():remote]
    depth = least = 0
    for ch in between:
        depth += {"{": 1, "}": -1}.get(ch, 0)
        least = min(least, depth)
    assert least == 0


def test_no_block_leaves_while_its_shared_memory_may_be_read():
    """After the first access to another CTA's shared memory every way out of the kernel leads over a cluster barrier."""
    body = kernel_body("paged8_evict.cu", "paged8_evict_kernel")
    remote = [m.start() for m in re.finditer(REMOTE, body)]
    ways_out = [m.start() for m in re.finditer(r"\breturn;", body)] + [len(body)]
    for out in (w for w in ways_out if w > remote[0]):
        before = [r for r in remote if r < out]
        assert re.search(START + r"|cluster_arrive|barrier\.cluster", body[before[-1]:out]), "a way out without a barrier"


def test_move_reads_before_it_writes():
    """A round's tokens have arrived before the CTA comes to the round's cluster barrier, and nothing of the cache is written
    before it has passed it: the places that one CTA writes may be what another one's loads of the same round read."""
    body = kernel_body("paged8_evict.cu", "paged8_evict_kernel")
    loop = body[body.index("for (; round < rounds; ++round)"):]
    arrived, arrive, wait = (loop.index(x) for x in ("cp_async_wait<kStages - 2>()", "barrier.cluster.arrive", "barrier.cluster.wait"))
    assert arrived < arrive < wait
    stores = [m.start() for m in re.finditer(r"reinterpret_cast<uint4\*>\(codes|scale\[[^;=]*\] =|mass\[[^;=]*\] =", body)]
    assert len(stores) == 3 and min(stores) > body.index("for (; round < rounds; ++round)") + wait
