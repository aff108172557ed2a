"""Training rounds whose input and weight gradients share a launch of more tiles than it has workgroups, and how they share them (not a test module):
(kind, jobs, (workgroups that add columns, that walk input gradients, that walk weight gradients))."""
from block_rounds import jobs

SPLITS = [
    # by whole tiles: a tile of each kind after the other divides evenly
    ("dense_train", [(500, 2048, 2048)] * 4, (128, 256, 256)),
    ("dense_train", jobs(16, 188, 1360, 1000), (256, 256, 256)),
    # by the work: both kinds walk
    ("dense_train", jobs(4, 500, 2048, 2048), (136, 200, 312)),
    ("dense_train", jobs(12, 313, 1320, 296), (64, 248, 264)),
    ("gated_train", jobs(16, 221, 800, 664, 504), (0, 184, 328)),
    # every input gradient's tile has a place, weight gradients walk
    ("dense_train", [(400, 768, 768)] * 10, (120, 240, 272)),
    ("gated_train", jobs(10, 166, 760, 368, 400), (0, 120, 392)),
]
