"""What a pass over trees' nodes says goes by the nodes alone: not by whether logits are asked for, nor by how many sequences the stage is for."""
import random

import numpy as np
import pytest
import torch

import continuations_plain as plain
import synth
from helpers import make_gpu, to_dev
from test_gpu_continuations import BF16, F32, GENERIC, WIDE, bounds

pytestmark = pytest.mark.gpu

NARROW = synth.StageShape("bf16", 1, 64, 1, 1, 64, 128, 130001)  # half a megabyte of logits a row, an odd number of them


@pytest.mark.parametrize("shape,nodes", [(s, n) for s in (F32, BF16, GENERIC, WIDE) for n in ([26], [5, 9, 2], [40, 64, 5])] + [(NARROW, [64, 64, 20]), (NARROW, [3, 9])],
                         ids=lambda x: str(x) if isinstance(x, list) else "%s_%d" % (x.dtype, x.vocab))
def test_what_is_said_with_logits_and_without(shape, nodes):
    r = random.Random(sum(nodes))
    lengths = [9, 30, 14][: len(nodes)]
    trees = [plain.random_tree(r, n) for n in nodes]
    st = make_gpu(shape, 3, 0, shape.n_layers_total, len(nodes), 110, 160)
    st.prefill(to_dev(shape, np.concatenate([synth.token_ids(20 + b, n, shape.vocab) for b, n in enumerate(lengths)])), lengths)
    parents, cu, host = bounds(trees)
    for seed in range(30, 40):
        feed = torch.from_numpy(np.concatenate([synth.token_ids(seed + b, n, shape.vocab) for b, n in enumerate(nodes)])).cuda()
        said, logits = st.tree(feed, parents, cu, host, max(lengths), want_logits=True)
        alone = st.tree(feed, parents, cu, host, max(lengths))
        torch.cuda.synchronize()
        assert torch.equal(said, logits.argmax(1).int())
        assert torch.equal(alone, said), (seed, (alone != said).nonzero().flatten().tolist())
    st.close()


def test_few_nodes_many_times():
    """As few nodes as the head's GEMM can take with the norm inside it: among a thousand tokens some have two logits next to each other."""
    r, nodes = random.Random(1), [5, 9, 2]
    st = make_gpu(BF16, 3, 0, 2, 3, 40, 60)
    parents, cu, host = bounds([plain.random_tree(r, n) for n in nodes])
    for seed in range(60):
        feed = torch.from_numpy(synth.token_ids(seed, 16, BF16.vocab)).cuda()
        said, _ = st.tree(feed, parents, cu, host, 0, want_logits=True)
        assert torch.equal(st.tree(feed, parents, cu, host, 0), said), seed
    st.close()


def test_a_pass_without_logits_reads_the_head_as_often_as_one_with_them():
    """A stage for one sequence, mostly head (0.5 GB: 100 us and more each time it is read), 40 nodes: read once, not once for each node."""
    shape = synth.StageShape("bf16", 1, 2048, 1, 1, 64, 128, 128000)
    st = make_gpu(shape, 3, 0, 1, 1, 80, 64)
    parents, cu, host = bounds([plain.random_tree(random.Random(2), 40)])
    feed = torch.from_numpy(synth.token_ids(5, 40, shape.vocab)).cuda()

    def fastest(**kw):
        times = []
        for _ in range(8):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            st.tree(feed, parents, cu, host, 0, **kw)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    fastest()
    assert fastest() <= 3 * fastest(want_logits=True)  # 30 times it where each node reads the head
    st.close()
