"""The plan of paged attention (lpp_paged_plan.h) on the host: the inputs of the GPU tests take the paths that they are for (no GPU)."""
import numpy as np
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


# dtype, H, Hkv, Dh, then the largest B, M, S and a smaller call's: what the workspace of the former alone used to be too short for
GROWN = [("bf16", 32, 8, 128, (2, 512, 3264), (2, 512, 3200)), ("bf16", 24, 8, 64, (16, 129, 4992), (16, 129, 4928)),
         ("bf16", 24, 24, 64, (8, 61, 2400), (1, 61, 2400)), ("bf16", 32, 8, 128, (64, 1, 900), (1, 1, 900)),
         ("f32", 16, 16, 64, (60, 16, 700), (2, 16, 600))]


@pytest.mark.parametrize("dtype,H,Hkv,Dh,largest,smaller", GROWN)
def test_a_workspace_serves_smaller_calls(plan, dtype, H, Hkv, Dh, largest, smaller):
    need = plan(dtype, smaller[0], H, Hkv, Dh, *smaller[1:]).bytes
    assert plan(dtype, largest[0], H, Hkv, Dh, *largest[1:]).bytes < need <= plan.room(dtype, largest[0], H, Hkv, Dh, *largest[1:])


@pytest.mark.parametrize("n_cu", [256, 64, 304])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_room_holds_every_plan_and_grows(plan, dtype, n_cu):
    rng = np.random.default_rng(n_cu)

    def size(most):
        return int(round(np.exp(rng.uniform(0, np.log(most)))))

    for _ in range(4000):
        Hkv, gq, Dh = size(64), size(16), int(rng.choice([64, 128]))
        at = [size(300), gq * Hkv, size(8192), size(200000) - 1]                # B, H, M, S
        room, p = plan.room(dtype, at[0], at[1], Hkv, Dh, at[2], at[3], n_cu), plan(dtype, at[0], at[1], Hkv, Dh, at[2], at[3], n_cu)
        assert p.bytes <= room < 2 ** 31 and (p.nsplit > 1) == (p.bytes > 0)
        for i in range(4):
            more = list(at)
            more[i] += size(at[i] + 2) * (Hkv if i == 1 else 1)
            assert plan.room(dtype, more[0], more[1], Hkv, Dh, more[2], more[3], n_cu) >= room, (at, more)
