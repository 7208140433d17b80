"""The plan of paged attention (lpp_paged_plan.h) on the host: the inputs of the GPU tests take the paths that they are for (no GPU)."""
import pytest

import paged_paths
import paged_plan


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    return paged_plan.build(tmp_path_factory.mktemp("paged_plan"))


def joining(p):
    return "one" if p.nsplit == 1 else "later" if p.join_later else "last"


@pytest.mark.parametrize("path", paged_paths.PATHS)
def test_inputs_take_their_path(plan, path):
    dtype, Dh, shape, joined, by_lengths, _, B, H, Hkv, M, S, _ = path
    p = plan(dtype, B, H, Hkv, Dh, M, S)
    assert (p.shape, joining(p), p.by_lengths) == (shape, joined, by_lengths), p
    assert p.range >= 2 * p.wk                             # (a wave has a second tile)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_whose_ranges_the_last_block_joins(plan, dtype):
    for lens in paged_paths.TOKENS:
        p = plan(dtype, len(lens), 8, 2, 128, 1, max(lens))
        assert joining(p) == "last" and p.nsplit > 4, p
