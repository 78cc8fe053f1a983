"""Compaction of pools of several thousand pages, which takes several rounds of 1024: holes and pages that fill them in one round, in far
ones and across a round's end; in place and into another pool.  Compared exactly."""
import random

import pytest
import torch

import paper_2603_19664_b200 as kvd
from test_gpu_cache4 import ints, open_ctx
from test_gpu_pages import Model, State, pages_of

pytestmark = pytest.mark.gpu
PAGE = kvd.KVD_PAGE_TOKENS


def used_pages(rng, kind, pages, used):
    """`used` page numbers of the pool."""
    if kind == "low":      # nothing to move
        return list(range(used))
    if kind == "high":     # everything above the count moves, and what is below it stays
        return list(range(pages - used, pages))
    if kind == "scattered":
        return rng.sample(range(pages), used)
    if kind == "one hole":  # the last page of the pool goes to a hole of the first round
        return [p for p in range(used) if p != 700] + [pages - 1]
    holes = list(range(900, 1023))  # "far": the holes lie in the first round, the pages that fill them in the last
    return [p for p in range(used) if p not in holes] + list(range(pages - len(holes), pages))


@pytest.mark.parametrize("kind", ["low", "high", "scattered", "one hole", "far"])
@pytest.mark.parametrize("pages,used", [(4500, 1023), (4500, 1024), (4500, 1025), (4096, 2048), (4500, 3000), (5121, 4097), (5121, 5121 - 123)])
def test_pools_of_many_rounds(pages, used, kind):
    ctx, desc = open_ctx("smollm2")
    rng = random.Random(pages + used)
    seqs, most = 40, 200
    st, m = State(desc, pages, seqs, most), Model(pages, seqs, most)
    held = used_pages(rng, kind, pages, used)
    assert len(set(held)) == used and max(held) < pages
    rng.shuffle(held)
    for s in range(seqs - 1):
        mine = held[s::seqs - 1]
        m.table[s][:len(mine)] = mine
        m.lens[s] = PAGE * len(mine) - (s if mine else 0)
        for p in mine:
            m.refs[p] += 1
    m.table[seqs - 1][:100], m.lens[seqs - 1] = held[:100], 100 * PAGE  # pages of others
    for p in held[:100]:
        m.refs[p] += 1
    st.table.copy_(torch.tensor(m.table, dtype=torch.int32))
    st.lens.copy_(torch.tensor(m.lens, dtype=torch.int32))
    st.refs.copy_(torch.tensor(m.refs, dtype=torch.int32))
    st.check(m)
    to = m.compact()
    assert sorted(to.values()) == list(range(used))
    scratch = torch.empty(kvd.kvd_pages_scratch_bytes(pages), dtype=torch.uint8, device="cuda")
    n_used = ints(0)

    def moved(model):
        for s in range(seqs):
            model.table[s][:pages_of(m.lens[s])] = [to[p] for p in m.held(s)]
        model.lens = list(m.lens)
        refs, tags = [0] * len(model.refs), list(model.tags)
        for p, d in to.items():
            refs[d], tags[d] = m.refs[p], m.tags[p]
        return refs, tags

    for room in (used, used + 37, pages + 500):
        new, nm = State(desc, room, seqs, most), Model(room, seqs, most)
        nm.refs, nm.tags = moved(nm)
        ctx.kvd_pages_compact(st.tuple, new.tuple, scratch, n_used)
        assert n_used.item() == used and ctx.kvd_poll_status() == 0
        new.check(nm)
        st.check(m)
    after = Model(pages, seqs, most)
    after.table = [list(row) for row in m.table]
    refs, tags = moved(after)
    after.refs, after.tags = refs, tags
    n_used.zero_()
    ctx.kvd_pages_compact(st.tuple, st.tuple, scratch, n_used)
    assert n_used.item() == used and ctx.kvd_poll_status() == 0
    st.check(after)
