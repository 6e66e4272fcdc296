"""Where a row stands in its sequence: calls without cu_seqlens whose tokens are not appended, and one cache in both roles.
Tolerances: those of test_gpu_prefix, whose definition in 64 bits this uses."""

import math

import pytest
import torch

from tests.test_gpu_prefix import Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch", [7, 40, 270], ids=["few", "wide", "table"])
@pytest.mark.parametrize("appended", [True, False], ids=["appended", "drafts"])
def test_one_token_each_without_cu(batch, appended):
    """Gates off, places around the edge of the window: a row at the wrong place sees one key too many or too few."""
    w = 16
    own = [(0 if not appended else 1, 1, 2, w - 2, w - 1, w, w + 1)[b % 7] for b in range(batch)]
    s = Setup([3, w - 1, w, 90], own, [b % 4 for b in range(batch)], 8, 2, 64, window=w, keep=0.0, seed=batch)
    q = s.randn(batch, 8, 64).bfloat16()
    part, part_lse = s.randn(batch, 8, 64).bfloat16(), s.randn(batch, 8)
    part_lse[0] = -math.inf
    ref = s.reference(q, [1] * batch, (part, part_lse), appended=appended)
    out, lse = s.cache.prefix_attention(s.sharing, q, None, part, part_lse, appended=appended)
    s.check(out, lse, ref, "cu None")
    out, lse = s.cache.prefix_attention(s.sharing, q, list(range(batch + 1)), part, part_lse, appended=appended)
    s.check(out, lse, ref, "cu given")
