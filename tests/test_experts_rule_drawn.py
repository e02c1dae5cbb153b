"""The choice of the tile (dash_experts_rule.h) on layers that its constants were not fitted to: the sixteen of 441 drawn layers that it serves worst
and sixteen others, with the times of every tile.  No GPU involved."""
import pytest

from test_experts_rule import lib, tile  # noqa: F401  (a fixture)

# 4-bit weights; rows, experts, K, M, primes; us of repeated calls with each tile (big, narrow; 4-bit also few, wide); the choice's over the least.
# Several of them have shares as uneven as 1 / (e + 1)^2, which the rule does not see.
DRAWN = [
    ((False, 24, 15, 1170, 570, 8), (20.0, 14.6), 1.37),
    ((False, 294, 62, 1417, 341, 7), (104.2, 76.7), 1.36),
    ((False, 104, 8, 467, 520, 12), (42.8, 34.9), 1.23),
    ((True, 8, 10, 3617, 744, 9), (47.2, 33.1, 27.5, 34.5), 1.20),
    ((True, 153, 19, 1473, 216, 9), (50.6, 47.9, 67.8, 42.5), 1.19),
    ((False, 20, 2, 359, 2869, 9), (30.0, 25.2), 1.19),
    ((False, 506, 16, 1185, 277, 9), (150.7, 132.3), 1.14),
    ((True, 8, 18, 155, 2236, 8), (16.9, 13.6, 19.4, 12.0), 1.13),
    ((True, 6, 3, 92, 2154, 12), (14.8, 12.2, 15.9, 10.8), 1.13),
    ((True, 50, 5, 3845, 794, 7), (96.0, 90.8, 123.3, 101.4), 1.12),
    ((False, 24, 18, 1212, 2763, 8), (55.1, 49.4), 1.12),
    ((True, 44, 39, 2915, 10, 9), (40.0, 21.0, 23.3, 30.3), 1.11),
    ((False, 440, 3, 1684, 191, 7), (85.6, 77.6), 1.10),
    ((True, 7, 7, 3916, 2229, 7), (51.5, 53.6, 54.0, 56.8), 1.10),
    ((False, 11, 7, 1714, 1909, 9), (27.1, 24.6), 1.10),
    ((True, 112, 7, 611, 1711, 8), (94.2, 103.2, 175.5, 85.7), 1.10),
    ((False, 9, 1, 359, 86, 12), (11.0, 6.3), 1.00),
    ((True, 8, 1, 1395, 232, 12), (21.6, 12.2, 10.5, 16.8), 1.00),
    ((True, 54, 2, 882, 474, 12), (35.1, 29.6, 42.2, 29.5), 1.00),
    ((True, 4, 16, 3911, 16, 7), (41.8, 23.1, 17.8, 33.7), 1.00),
    ((True, 65, 1, 1846, 1130, 9), (84.3, 88.4, 131.0, 84.9), 1.01),
    ((True, 22, 2, 3226, 35, 8), (41.9, 21.1, 17.3, 30.7), 1.00),
    ((True, 96, 9, 1619, 25, 7), (28.2, 19.5, 24.0, 29.9), 1.00),
    ((True, 46, 2, 945, 3945, 7), (102.9, 114.1, 183.3, 91.8), 1.00),
    ((False, 1, 1, 1024, 374, 9), (15.6, 7.6), 1.00),
    ((False, 4, 28, 2600, 10, 12), (27.1, 11.2), 1.00),
    ((True, 940, 1, 2558, 19, 7), (234.2, 141.2, 208.4, 222.7), 1.00),
    ((True, 1, 2, 2638, 48, 12), (30.4, 17.1, 13.5, 24.7), 1.00),
    ((False, 96, 3, 3486, 391, 12), (86.8, 94.1), 1.00),
    ((True, 165, 29, 776, 63, 8), (34.8, 21.8, 30.1, 28.4), 1.00),
    ((True, 28, 2, 325, 1897, 9), (33.9, 29.4, 45.0, 25.4), 1.00),
    ((True, 236, 17, 166, 121, 9), (27.8, 15.1, 26.2, 20.5), 1.00),
]


@pytest.mark.parametrize("layer,times,over", DRAWN)
def test_what_the_choice_costs(lib, layer, times, over):  # noqa: F811
    mx4, rows, experts, K, M, k = layer
    assert len(times) == (4 if mx4 else 2)
    assert times[tile(lib, rows, experts, K, M, mx4, k) - 1] / min(times) <= over + 0.005
