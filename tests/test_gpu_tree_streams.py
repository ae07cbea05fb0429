"""A pass over trees between work on torch's current stream, on the null stream and on a stream given by hand."""
import random

import numpy as np
import pytest
import torch

import continuations_plain as plain
import synth
from helpers import make_gpu, to_dev
from test_gpu_continuations import F32, bounds

pytestmark = pytest.mark.gpu

LENGTHS, NODES, LONG = [9, 30], [7, 5], 40_000_000  # about 20 ms


def ready():
    st = make_gpu(F32, 3, 0, 2, 2, 60, 60)
    parents, cu, host = bounds([plain.random_tree(random.Random(n), n) for n in NODES])
    feeds = [torch.from_numpy(synth.token_ids(i, sum(NODES), F32.vocab)).cuda() for i in range(3)]
    prompt = to_dev(F32, np.concatenate([synth.token_ids(20 + b, n, F32.vocab) for b, n in enumerate(LENGTHS)]))
    st.prefill(prompt, LENGTHS)
    want = [st.tree(f, parents, cu, host, 30) for f in feeds]
    torch.cuda.synchronize()
    return st, parents, cu, host, feeds, prompt, [w.tolist() for w in want]


@pytest.mark.parametrize("by_hand", [False, True], ids=["current", "given"])
def test_the_whole_step_on_a_stream_of_its_own(by_hand):
    """Drafts that arrive late on the current stream; acceptance and compaction behind the pass."""
    from paper_2502_09922_amd import tree_accept, tree_keep

    st, parents, cu, host, feeds, _, want = ready()
    (k, v), side = st.caches(), torch.cuda.Stream()
    lens, feed = st.seq_lens.clone(), feeds[0].clone()
    torch.cuda.synchronize()
    for i in (1, 2, 0):
        with torch.cuda.stream(side):
            st.seq_lens.copy_(lens)
            torch.cuda._sleep(LONG)
            feed.copy_(feeds[i])
            said = st.tree(feed, parents, cu, host, 30, stream=side if by_hand else None)
            kept, count, emitted, following = tree_accept(feed, said, parents, cu, host)
            tree_keep(kept, cu, host, k, v, st.seq_lens)
        side.synchronize()
        assert said.tolist() == want[i]
        assert st.seq_lens.tolist() == (lens + count).tolist() and emitted[:, 0].tolist() == [want[i][0], want[i][NODES[0]]]
    st.close()


def test_between_passes_on_the_null_stream():
    """A prompt in front and a generation step behind, both on the null stream."""
    st, parents, cu, host, feeds, prompt, want = ready()
    side = torch.cuda.Stream()
    st.seq_lens.zero_()
    st.k.zero_()
    torch.cuda.synchronize()
    torch.cuda._sleep(LONG)
    st.prefill(prompt, LENGTHS)
    with torch.cuda.stream(side):
        said = st.tree(feeds[0], parents, cu, host, 30)
        late = [st.tree(f, parents, cu, host, 30) for f in feeds]
    st.decode(said[:2], 2, 30)
    torch.cuda.synchronize()
    assert said.tolist() == want[0] and [x.tolist() for x in late] == want
    assert st.seq_lens.tolist() == [n + 1 for n in LENGTHS]
    st.close()


def test_inputs_that_are_let_go_at_once():
    """On a stream that is not the current one, behind work that takes long: what the call was given is not handed out again before it has run."""
    st, parents, cu, host, feeds, _, want = ready()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in (0, 1, 2):
        with torch.cuda.stream(side):
            torch.cuda._sleep(LONG)
        made = [feeds[i].clone(), parents.clone(), cu.clone()]
        side.wait_stream(torch.cuda.current_stream())
        out = st.tree(*made, host, 30, stream=side)
        del made
        for _ in range(20):  # whoever gets their memory writes there
            torch.zeros_like(feeds[i]), torch.zeros_like(parents), torch.zeros_like(cu)
        side.synchronize()
        assert out.tolist() == want[i]
    st.close()


def test_captured_on_the_current_stream():
    st, parents, cu, host, feeds, _, want = ready()
    feed, graph = feeds[0].clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        said = st.tree(feed, parents, cu, host, 30)
    for i in (2, 0, 1, 1):
        feed.copy_(feeds[i])
        graph.replay()
        torch.cuda.synchronize()
        assert said.tolist() == want[i]
        assert st.tree(feed, parents, cu, host, 30).tolist() == want[i]
    st.close()
