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
