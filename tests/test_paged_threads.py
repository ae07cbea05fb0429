"""A PagedCache that several threads call at once: each gets the plan of its own call."""
import sys
import threading

import torch

from paper_2502_09922_amd import binding as b

HERE = 4096  # an aligned address that no query looks at


def cache():
    """What PagedCache makes of tensors on a GPU, as far as plans of calls go by it."""
    c = object.__new__(b.PagedCache)
    c._t = dict(k=torch.empty(1, 300, 2, 16, 64, dtype=torch.bfloat16, device="meta"))
    c._all = b.ls_pages(HERE, HERE, HERE, HERE, HERE, HERE + 4096, HERE, 300, 16, 300)
    c._heads, c._call, c.batch = {}, None, 3
    return c


def test_plans_of_calls_at_once():
    """Layers, contexts, tables of angles and numbers of query heads of their own: with another call's plan a kernel would take rows
    for longer than they are, or scratch for larger."""
    calls = [((8 + 4) * 64, 5000, 100), ((8 + 4) * 64, 5000, 4000), ((4 + 4) * 64, 5000, 100), ((8 + 4) * 64, 200, 100)]
    want = []
    for columns, max_seq, max_ctx in calls:
        hq, heads, nb = cache().attention_call(columns, max_seq, max_ctx)
        want.append((hq, heads.n_q_heads, heads.max_seq, nb))
    assert len(set(want)) == len(want) and [w[0] for w in want] == [8, 8, 4, 8] and all(w[3] for w in want)
    one, wrong, start = cache(), [], threading.Barrier(len(calls))

    def caller(call, own):
        start.wait()
        for _ in range(20000):
            hq, heads, nb = one.attention_call(*call)
            if (hq, heads.n_q_heads, heads.max_seq, nb) != own:
                wrong.append((call, hq, heads.max_seq, nb))

    before = sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    try:
        threads = [threading.Thread(target=caller, args=x) for x in zip(calls, want)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(before)
    assert not wrong, (len(wrong), wrong[:3])
