"""How far the warps of the chunk weights' kernel may run ahead of one another, and that its barriers are told apart over that
distance: a wait by parity misses a phase where the barrier completes twice before the waiting warp has looked."""
import os
import re

import pytest

from paper_2607_15498_gb300 import build
from test_source_order import kernel_body


def source(file):
    return re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, file)).read())


def ahead_of(held, scores, lse, units=40):
    """Units of one query tile each, dealt to two key tiles, whose sums two halves of warps add up: the second half hands its sum over
    (the barrier `half`), the first waits for that. With the first half of key tile `held` standing before its wait of unit 0,
    everything else runs as far as it may: how many more times the barrier of that tile has completed."""
    done = {}                                    # (tile, unit, half): this half has given the scores of a unit back
    product = set()
    halves = [0, 0]                              # completions of the barrier by key tile
    waits = {(e, h): 0 for e in (0, 1) for h in (0, 1)}
    moved = True
    while moved:
        moved = False
        for e in (0, 1):
            for n in range(units):               # the place of product 2 n + e is that of the product `scores` before it
                j = 2 * n + e - scores
                free = j < 0 or all(done.get((j & 1, j >> 1, h)) for h in (0, 1))
                if (e, n) not in product and (n == 0 or (e, n - 1) in product) and free:
                    product.add((e, n))
                    moved = True
        for e, h in waits:
            n = waits[e, h]
            if n >= units or (e, n) not in product or (e == held and h == 0):
                continue
            # the rows' sums of a unit are fetched when all warps have given back those of `lse` units before
            if n >= lse and not all(done.get((x, n - lse, y)) for x in (0, 1) for y in (0, 1)):
                continue
            if h:
                halves[e] += 1
            elif halves[e] <= n:
                continue
            done[e, n, h] = True
            waits[e, h] = n + 1
            moved = True
    assert halves[held] >= 1
    return halves[held] - 1


@pytest.mark.parametrize("held", [0, 1])
def test_half_sums_are_told_apart(held):
    text = source("paged8_mass_tc.cu")
    scores, lse = (int(re.search(rf"\b{name} = (\d+)", text).group(1)) for name in ("kScores", "kLse"))
    declared = re.search(r"\bhalf_full\[2\](?:\[(\w+)\])?", text).group(1) or "1"
    n = int(declared) if declared.isdigit() else int(re.search(rf"\b{declared} = (\d+)", text).group(1))
    assert n > ahead_of(held, scores, lse), "the barrier may complete a second time before the first half has seen it"
    # by the number of the unit, and the parity by how often that barrier has been used
    uses = re.findall(r"(mbar_arrive|warp_wait)\(&c\.half_full\[e\]([^,)]*)(?:, ([^)]*\)[^)]*))?\)", text)
    assert [u[0] for u in uses] == ["mbar_arrive", "warp_wait"]
    index = {f"[un % {declared}]", f"[un & {n - 1}]"} if n > 1 else {""}
    assert uses[0][1] == uses[1][1] and uses[0][1] in index
    assert uses[1][2] in (f"(un / {declared}) & 1", f"(un >> {n.bit_length() - 1}) & 1")


@pytest.mark.parametrize("file, kernel", [("paged8_append.cu", "paged8_append_kernel"), ("paged8_attn.cu", "paged8_attn_kernel"),
                                          ("paged8_attn_tc.cu", "paged8_attn_tc_kernel"), ("paged8_merge.cu", "paged8_merge_kernel"),
                                          ("paged8_mass.cu", "paged8_mass_kernel"), ("paged8_mass_tc.cu", "paged8_mass_tc_kernel"),
                                          ("paged8_evict.cu", "paged8_evict_kernel")])
def test_every_kernel_waits_before_it_reads(file, kernel):
    """Kernels are launched while the one before still runs: each waits for it whatever its arguments, before anything in memory that
    another kernel may have written is looked at. That the one before has waited in its turn is not enough."""
    body = kernel_body(file, kernel)
    wait = body.index("pdl_wait()")
    before = body[:wait]
    assert before.count("{") == before.count("}") and re.search(r"[;}]\s*$", before) and not re.search(r"\belse\s*$", before)
    assert not re.search(r"__ldg|header->|table\[|seq_range|plan_\w+<|\bkv_len\b|row_start|tma_load|\bscale\[|\bmass\[", before)
    assert body.count("pdl_wait()") == 1
