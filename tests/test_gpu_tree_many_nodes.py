"""fp32 passes over more nodes than a generation step has rows: their projections take the GEMMs that a prompt pass of as many rows takes."""
import random

import numpy as np
import pytest
import torch

import continuations_plain as plain
import synth
from helpers import check_close, make_gpu, make_oracle, to_dev, to_host
from test_gpu_continuations import bounds

pytestmark = pytest.mark.gpu


def test_a_pass_takes_about_what_a_prompt_of_as_many_rows_takes():
    """640 rows of 8192 columns, whose partial tiles need 20 MiB: with the O and down projections by the generic kernel 3.7 ms, the prompt 1.4."""
    shape = synth.StageShape("f32", 1, 8192, 64, 8, 128, 2048, 0)
    st = make_gpu(shape, 3, 0, 1, 10, 70, 640)
    parents, cu, host = bounds([plain.random_tree(random.Random(b), 64) for b in range(10)])
    x = torch.randn(640, 8192, device="cuda")

    def fastest(call):
        times = []
        for _ in range(6):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            st.seq_lens.zero_()
            a.record()
            call()
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    tree, prompt = (lambda: st.tree(x, parents, cu, host, 0)), (lambda: st.prefill(x, [64] * 10))
    fastest(tree), fastest(prompt)
    assert fastest(tree) <= 1.6 * fastest(prompt)
    st.close()


def test_rows_of_many_nodes_are_those_of_prompt_passes():
    """A chain in each tree: its rows are a prompt's."""
    shape = synth.StageShape("f32", 1, 4096, 4, 2, 128, 512, 0)
    x = synth.hidden_states(shape, 6, 1100)
    trees = [list(range(-1, 63)) for _ in range(17)] + [list(range(-1, 11))]
    st = make_gpu(shape, 3, 0, 1, 18, 70, 1100)
    parents, cu, host = bounds(trees)
    got = st.tree(to_dev(shape, x), parents, cu, host, 0)
    want = make_oracle(shape, 3, 0, 1, 18, 70).prefill(x, [len(t) for t in trees])
    check_close(to_host(got), want, "f32", "many nodes")
    assert np.array_equal(host, np.cumsum([0] + [len(t) for t in trees]))
    st.close()
