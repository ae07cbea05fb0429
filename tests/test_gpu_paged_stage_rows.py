"""A stage with room for more sequences than a cache in pages has: whose rows of lens and positions lie side by side, or as near as small
allocations do."""
import numpy as np
import pytest
import torch

import synth
from helpers import make_gpu, to_dev

pytestmark = pytest.mark.gpu

F32 = synth.CONFIGS["tiny_f32"]
BF16 = synth.StageShape("bf16", 2, 512, 8, 2, 128, 1408, 1000)
LENGTHS = [9, 20]


def steps(shape, max_batch, marks, weighed):
    """Three steps of a stage with `max_batch` places over a cache of two sequences whose lens and positions `marks` makes."""
    from paper_2502_09922_amd import PagedCache, paged_fill

    st = make_gpu(shape, 3, 0, 2, max_batch, 40, 200)
    prompt = to_dev(shape, np.concatenate([synth.token_ids(20 + b, n, shape.vocab) for b, n in enumerate(LENGTHS)]))
    said = st.prefill(prompt, LENGTHS)
    k, _ = st.caches()
    size = (k.shape[0], 8, k.shape[2], 8, k.shape[4])
    pools = [torch.zeros(size, dtype=k.dtype, device="cuda") for _ in "kv"]
    more = [torch.zeros(size[:-1], device="cuda"), torch.zeros(size[:-1], dtype=torch.int32, device="cuda")] if weighed else [None, None]
    lens, positions = marks()
    table = torch.tensor([[5, 2, 0, 7], [1, 6, 3, 4]], dtype=torch.int32).cuda()
    cache = PagedCache(*pools, table, lens, positions, *more)
    paged_fill(cache, *st.caches(), st.seq_lens, torch.arange(2, dtype=torch.int32).cuda(), 20)
    found = []
    for step in range(3):
        said, logits = st.paged(said, cache, 20 + step, want_logits=True)
        found.append(logits.clone())
    torch.cuda.synchronize()
    assert lens.tolist() == positions.tolist() == [12, 23]
    st.close()
    return found


@pytest.mark.parametrize("weighed", [False, True], ids=["", "weighed"])
@pytest.mark.parametrize("shape", [F32, BF16], ids=["f32", "bf16"])
def test_a_stage_with_more_places_than_the_cache_has_sequences(shape, weighed):
    def far():
        return torch.zeros(2, 1000, dtype=torch.int32, device="cuda")[:, :2].unbind()

    def rows():
        return torch.zeros(2, 2, dtype=torch.int32, device="cuda").unbind()

    def near():  # two allocations of the smallest size
        return torch.zeros(2, 128, dtype=torch.int32, device="cuda")[:, :2].unbind()

    for max_batch in (2, 3, 8, 129, 200):
        want = steps(shape, max_batch, far, weighed)
        for marks in (rows, near):
            for a, b in zip(steps(shape, max_batch, marks, weighed), want):
                assert torch.equal(a, b), (max_batch, marks.__name__)


def test_one_buffer_is_refused():
    from paper_2502_09922_amd import LsError

    def twice():
        lens = torch.zeros(3, dtype=torch.int32, device="cuda")
        return lens[:2], lens[1:]

    with pytest.raises(LsError, match="one buffer"):
        steps(F32, 2, twice, False)
