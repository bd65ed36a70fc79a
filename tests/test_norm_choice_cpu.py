"""How the group norm cuts its work up (csrc/tdc_norm_choice.h), at the largest sizes that a plan takes."""
import pytest

import norm_choice

LARGEST = 2 ** 31 - 1
# H x W up to the largest product that a plan takes; 46340 x 46341 is within a chunk of it
IMAGES = [(1, LARGEST), (1, LARGEST - 300), (46340, 46341), (2, 2 ** 30 - 1), (1, 2 ** 31 - 2 ** 21), (1, 2 ** 30 + 1), (1, 2 ** 24)]


@pytest.mark.parametrize("batch", [1, 2, 3, 700, 1024, 65535])
@pytest.mark.parametrize("H,W", IMAGES)
def test_chunks_of_the_largest_images(H, W, batch):
    """They cover the image, none is empty, and the workspace counts what the launches write."""
    P = H * W
    for C, groups in ((1, 1), (8, 2), (8192, 32)):
        for size in (2, 4):
            c = norm_choice.chunks((batch, H, W, C, groups), size)
            assert 1 <= c["chunks"] <= 1024 and 1 <= c["chunk_px"] <= P
            assert (c["chunks"] - 1) * c["chunk_px"] < P <= c["chunks"] * c["chunk_px"]
            assert c["images"] * c["chunks"] <= c["sum_rows"] <= 1024


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("H,W", IMAGES)
def test_no_image_of_that_size_stays_in_registers(H, W, backward):
    for C, groups, V in ((1, 1, 1), (2, 1, 2), (8, 2, 4), (8, 8, 1), (64, 32, 4), (8192, 8192, 4)):
        assert norm_choice.slices((1, H, W, C, groups), 4, V, backward)["held"] == 0


# B, H, W, C, groups, bytes to an element, channels to an access: slices that would be widened by 1024 threads or not, and pass 2^32
MANY = [(65535, 746, 1, 715, 715, 2, 1), (65535, 1, 130, 4020, 1340, 2, 1), (65535, 149, 1, 3536, 884, 2, 1), (65535, 1, 1, 8144, 509, 4, 4), (40000, 700, 1, 1430, 715, 2, 1)]


@pytest.mark.parametrize("case", MANY)
def test_a_launch_has_fewer_than_2_32_threads(case):
    B, *rest, size, V = case
    cut = norm_choice.slices((B, *rest), size, V)
    assert B * cut["slices"] * cut["threads"] < 2 ** 32
    assert B * norm_choice.chunks((B, *rest), size)["chunks"] * 512 < 2 ** 32
