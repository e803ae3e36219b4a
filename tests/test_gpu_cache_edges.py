"""Attention weight per slot and eviction where a call's parts are missing, infinite or laid out backwards, against
the same call on whole inputs or their plain forms in 64 bits (tests/cache_reference.py, which states the
tolerances)."""
from __future__ import annotations

import numpy as np
import pytest

from test_gpu_cache import BAD_LAYOUT, call_mass, check_mass, mass_inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch

    import paper_2609_14636_gb300 as stride

    return torch, stride, torch.device("cuda")


# ---------------------------------------------------------------------------------------------------------------------
# attention weights
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("page", [128, 256, 16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new", [13, 90], ids=["52 rows", "360 rows"])
@pytest.mark.parametrize("lost", ["first", "last", "all of one", "all", "many"])
def test_tiles_without_pages(env, page, D, new, lost):
    """Whole tiles of 128 slots have no page, in a call of several tiles for each CTA: NaN there, all other slots as if the
    pages were there (a slot's sum is its own: the same bits)."""
    torch, stride, dev = env
    case = ([(20000, new), (700, new), (0, new), (130, new)], 32, 8, D, page, "rows", False, 0.9, "bf16")
    x = mass_inputs(torch, case)
    before = x["mass"].clone()
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    call_mass(stride, torch, x, case, status)
    assert int(status) == 0
    whole = x["mass"].double().cpu().numpy()
    check_mass(x, case, before.double().cpu().numpy(), whole, skip=(0,))
    # the pages of those runs of 128 slots (or of a page, where it is longer)
    run, rng = max(128, page), np.random.default_rng(page)
    total = [c + n for c, n in case[0]]
    runs = [(b, r) for b, t in enumerate(total) for r in range(-(-t // run))]
    gone = {"first": [(0, 0)], "last": [(3, -(-total[3] // run) - 1), (0, -(-total[0] // run) - 1)],
            "all of one": [r for r in runs if r[0] == 1], "all": runs,
            "many": [r for r in runs if rng.random() < 0.5]}[lost]
    nan = np.zeros(whole.shape, bool)
    for b, r in gone:
        x["table"][b, r * run // page:(r + 1) * run // page] = (-1, len(x["k"]), 2 ** 31 - 1)[r % 3]
        nan[b, :, r * run:min((r + 1) * run, total[b])] = True
    for _ in range(3):
        m = before.clone()
        status.zero_()
        call_mass(stride, torch, x, case, status, m)
        assert int(status) == BAD_LAYOUT
        got = m.double().cpu().numpy()
        assert np.isnan(got[nan]).all() and np.array_equal(got[~nan], whole[~nan])
