"""Workgroups of the step's gradient, as its workspace has room for their sums (host code: no GPU needed)."""
import pytest

from paper_2605_17633_amd import binding as B


def workgroups(images, N, D, gate_images):
    """of a group of tokens: four vectors of D sums for each, and a place for the group's own where there are many"""
    room = B.ssam_residual_norm_backward_workspace_bytes(images, N, D, gate_images)
    assert room % (gate_images * 16 * D) == 0
    return room // (gate_images * 16 * D) - (gate_images > 1)


@pytest.mark.parametrize("D", [520, 1024, 1280, 1536, 1544, 2048])
def test_wide_rows_take_a_round(D):
    """A CU holds one workgroup of rows above 512: with more than 256 of them in all, the last few would run alone for as long as the others."""
    for images in range(1, 257):
        n = workgroups(images, 1 << 20, D, images)
        assert n >= 1 and images * n <= 256 and images * (n + 1) > 256
    assert workgroups(1000, 64, D, 1000) == 1 and workgroups(7, 1 << 20, D, 1) == 256


@pytest.mark.parametrize("D", [8, 128, 136, 256, 264, 512])
def test_narrow_rows_take_a_round_of_two(D):
    for images in range(1, 257):
        n = workgroups(images, 1 << 20, D, images)
        assert n >= 1 and images * n <= (256 if images <= 128 or images == 256 else 512)


@pytest.mark.parametrize("images,N,D", [(1, 1, 64), (3, 1, 2048), (5, 17, 1280), (200, 9, 144), (300, 1, 512)])
def test_no_more_than_there_are_tokens_for(images, N, D):
    lanes, waves = 16 if D <= 128 else 32 if D <= 256 else 64, 4 if D > 1536 else 8
    for gate_images in {1, images}:
        tokens, rows = images * N // gate_images, waves * 64 // lanes
        assert workgroups(images, N, D, gate_images) <= -(-tokens // rows)


@pytest.mark.parametrize("images,N,D,each", [(3, 1500, 1280, False), (3, 1500, 1280, True), (3, 6000, 64, False), (3, 6000, 144, True), (3, 1400, 2048, False), (5, 700, 520, True), (7, 500, 1280, True),
                                             (129, 40, 144, True), (129, 20, 1024, True), (6, 300, 2048, True)])
def test_sums_are_of_few_roundings(images, N, D, each):
    """What the bounds of the weights' gradients count for sums over tokens, 64 roundings beside the 100 of a term: a wave's tokens one after the other, the waves' shares of a workgroup,
    workgroups in 32 slices, five additions over those, and, of many groups, those in 32 slices and five more.  Nothing that the tests run has more."""
    groups = images if each else 1
    n, lanes, waves = workgroups(images, N, D, groups), 16 if D <= 128 else 32 if D <= 256 else 64, 4 if D > 1536 else 8
    shares = waves * 64 // lanes
    roundings = -(-(images * N // groups) // (n * shares)) + shares + -(-n * groups // 32) + 5 + (-(-groups // 32) + 5 if groups > 1 else 0)
    assert roundings <= 64, roundings
