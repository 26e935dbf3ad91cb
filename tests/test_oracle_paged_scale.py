"""The oracle of the paged append where a page's scale lies above the largest that an append gives."""
import numpy as np

from oracle import paged as P


def test_oracle_keeps_a_scale_above_its_largest():
    codes = np.full((4, 2), 100, dtype=np.int8)
    now = P.append_page(codes, np.float32(1.5 * 2.0 ** 120), 2, np.full((1, 2), 3.3e38, np.float32), "int8")
    assert now == np.float32(1.5 * 2.0 ** 120) and codes[:3].tolist() == [[100, 100], [100, 100], [127, 127]]
