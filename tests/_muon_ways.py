"""Sizes that take every kind of Newton-Schulz tiles: (matrices, shorter side, longer side): how the Gram matrix, the polynomial and the step are
computed, as (tile, in parts).  test_muon_plan.py compares them with the rule, test_gpu_muon_ways.py runs them."""
WAYS = {
    (1, 69, 69): ((64, False), (64, False), (64, False)),
    (1, 69, 741): ((64, True), (64, False), (64, False)),
    (8, 193, 871): ((128, True), (64, False), (64, False)),
    (8, 260, 802): ((192, True), (64, False), (128, False)),
    (8, 389, 839): ((256, True), (64, False), (128, False)),
    (8, 129, 4292): ((64, True), (64, False), (256, False)),
    (8, 641, 641): ((128, False), (128, False), (64, False)),
    (8, 962, 962): ((192, False), (192, False), (128, False)),
    (8, 1345, 1345): ((256, False), (256, False), (128, False)),
    (1, 1089, 1093): ((128, True), (128, True), (64, False)),
    (2, 1090, 1091): ((192, True), (192, True), (128, False)),
    (3, 1089, 1089): ((256, True), (256, True), (128, False)),
    (1, 1026, 3960): ((128, True), (64, False), (256, True)),
    (3, 1827, 2590): ((256, True), (192, False), (128, True)),
    (1, 69, 16532): ((64, True), (64, False), (128, False)),
    (1, 259, 21852): ((64, True), (64, False), (256, False)),
}
ALL = {(tile, parts) for tile in (64, 128, 192, 256) for parts in (False, True)}
# what the rule can pick: 64 x 64 in parts for Gram matrices alone, 192 for symmetric products
PICKED = (ALL, ALL - {(64, True)}, {(64, False), (128, False), (128, True), (256, False), (256, True)})
