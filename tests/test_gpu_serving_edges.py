"""The serving operators on the GPU where their parts meet: items of one block, pages that are missing, entries that nobody
sees, values that are not finite, scores far from zero. Definitions and tolerances are those of the operators' other tests."""
import numpy as np
import pytest
import torch

from tests.test_gpu_serving import NAN, T, _attend, _bound, _cache, _check_attention, _evict_reference, _moa, _rows_of, _slots, _trees, _word  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dh,hkv,hq,n", [(128, 2, 4, 20), (64, 3, 48, 17)])
def test_tree_items_of_one_block(dh, hkv, hq, n):
    """Stretches of several short items, the first of one block of positions: the queries of the second item may be there
    before its keys are asked for."""
    moa, rng = _moa(), np.random.default_rng(dh)
    lens = [int(x) for x in rng.integers(1, 128 - n, 40)]
    c = _cache(rng, "bf16", lens, hkv, dh, 16, 600)
    q, kn, vn = _rows_of(rng, "bf16", 40, n, hq, hkv, dh)
    _, _, mask = _trees(rng, 40, n, 0)
    out = moa.moa_paged_attention(c, q, kn, vn, mask=mask)
    torch.cuda.synchronize()
    _check_attention(c, "bf16", q, kn, vn, mask.cpu().numpy(), out, lens, n)
    for _ in range(50):
        assert torch.equal(moa.moa_paged_attention(c, q, mask=mask), out)
