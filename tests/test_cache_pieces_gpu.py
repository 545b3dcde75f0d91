"""Tree attention: blocks that several CTAs share, and blocks that one CTA finishes, in one CTA's run.  Values and tolerances
as in test_cache_gpu.py."""
import gc

import pytest

from test_cache_gpu import Case, sh, tree_mask  # noqa: F401  (sh: the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def nothing_left():
    """The modules behind this one find the device's memory as it was: frames that an exception's traceback keeps alive go, too."""
    yield
    gc.collect()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,g", [(1, 4), (7, 4), (31, 8), (33, 4)])     # a tile of rows, and two
def test_parts_of_a_block_before_whole_ones(sh, d, n, g, dt):
    """A CTA hands its part of a long context to the workspace and goes on with short contexts that it finishes itself: both leave through
    the same shared memory.  Copies beside them keep the memory busy, so that the parts' copies take their time."""
    lens = ([2500 + 37 * n, 3, 0, 130, 11] + [60, 1] * 3) * 11
    c = Case(91, lens, n, 2, g, d, 16, dt, mask=tree_mask(n))
    first = {k: v.clone() for k, v in c.run(sh).items()}
    assert not first["status"].any()
    c.check(first)
    busy, side = torch.empty(1 << 28, dtype=torch.uint8, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(30):
        if i % 5 == 0:
            with torch.cuda.stream(side):
                for _ in range(4):
                    busy[: 1 << 27].copy_(busy[1 << 27:])
        again = c.run(sh)
        for key in first:
            assert torch.equal(again[key], first[key])
    torch.cuda.synchronize()


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,g,shared", [(31, 8, 0), (40, 4, 130), (70, 3, 0), (7, 4, 0), (1, 8, 40)])
def test_values_that_are_no_numbers_in_one_and_two_tiles_of_rows(sh, d, n, g, shared, dt):
    """Every row that sees such a node gets it, whichever of a block's tiles of rows it is in; the other rows keep their bits."""
    sees = tree_mask(n)
    c = Case(17, [97, 200, 1, 128 - n // 2], n, 2, g, d, 16, dt, shared=shared, mask=sees)
    clean = {k: v.clone() for k, v in c.run(sh).items()}
    c.check(clean)
    kept = c.vc.clone()
    for node in sorted({0, n // 3, n - 1}):
        hit = torch.from_numpy(sees[:, node]).cuda()
        for bad in (float("nan"), float("inf"), -float("inf")):
            for i, x in enumerate(c.lens_list):
                c.vc[int(c.table[i][(x + node) // 16]), (x + node) % 16, 1, d - 3] = bad
            for _ in range(5):
                got = c.run(sh)
                seen = got["out"][:, hit][:, :, g:, d - 3].float()
                assert bool(seen.isnan().all() if bad != bad else (seen == bad).all())
                assert torch.equal(got["out"][:, ~hit], clean["out"][:, ~hit]) and torch.equal(got["lse"], clean["lse"])
                assert torch.equal(got["out"][:, :, :g], clean["out"][:, :, :g])
                assert torch.equal(got["out"][..., : d - 3], clean["out"][..., : d - 3])
            c.vc.copy_(kept)
