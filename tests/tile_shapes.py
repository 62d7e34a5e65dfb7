"""Ragged sizes at which every product of the feed-forward block and of the 8-bit projection takes every tile, each with a
reduction of at least 2 x stages + 1 parts (so that the pipelined loop turns) and, where it may be split, whole and in
ranges. test_launches.py holds the lists to that; the device tests run them."""

FEED_TILES = [          # rows, in_features, hidden_features, out_features
    (918, 467, 585, 668), (262, 9, 6625, 527), (13629, 270, 149, 12), (8696, 298, 748, 352), (5400, 1052, 194, 287), (1693, 447, 2178, 61),
    (2133, 18, 6962, 359), (13032, 10, 668, 343), (5383, 2721, 161, 16), (417, 2847, 2036, 46), (5549, 164, 2602, 123), (2014, 12, 267, 2999),
    (6191, 1212, 646, 251), (2405, 52, 2203, 2454), (15444, 10, 299, 825), (5830, 9, 4188, 196), (1073, 52, 5941, 3758), (169, 3230, 6101, 82),
    (2033, 29, 3575, 1082), (12716, 18, 6495, 77), (1661, 1176, 4365, 18)]
INT8_TILES = [          # rows, in_features, out_features
    (94, 1088, 10), (676, 788, 3055), (11541, 705, 285), (1007, 2184, 6124), (7546, 612, 779), (5206, 587, 2363), (1999, 1100, 1347)]
