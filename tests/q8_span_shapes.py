"""Shapes of window and tree calls that are meant for one kernel in one role, shared by the tests that run them and the one that
asks the launch plan whether they take it."""

from collections import namedtuple

# cols: query columns of a tile (16 split kernel, 64 wide, 128 and 256 prompt kernel); most: splits of the longest sequence
Shape = namedtuple("Shape", "name H Hq lens n window sinks cols most")

# two splits of the prompt kernel and more, whose records a merge joins
SPLIT_TREES = [
    Shape("16 slots of 64 drafts", 4, 28, [3000 - 11 * b for b in range(16)], [64 - b % 3 for b in range(16)], 0, 0, 256, 2),
    Shape("4 slots of up to 256 drafts", 4, 32, [5000, 4700, 5003, 4990], [256, 250, 255, 251], 0, 0, 256, 2),
    Shape("the same in a layer with a window", 4, 32, [7000, 6700, 9003, 6990], [256, 250, 255, 251], 4500, 70, 256, 2),
    Shape("one long slot of 3", 4, 28, [1500, 300, 333], [200, 190, 200], 0, 0, 128, 3),
    Shape("one long slot of 3 in a layer with a window", 4, 28, [2500, 300, 333], [200, 190, 200], 1200, 5, 128, 3),
]
SPLIT_WINDOWS = [
    Shape("4 chunks of 512", 2, 16, [6000, 5900, 6003, 5800], [512, 500, 512, 511], 4096, 64, 256, 2),
    Shape("one long chunk of 3", 4, 28, [1500, 300, 333], [200, 190, 200], 1200, 5, 128, 3),
]
# pages that no row sees, in each kernel
HIDDEN_WINDOWS = [
    Shape("split", 1, 7, [2000], [1], 300, 10, 16, 1),
    Shape("wide", 1, 16, [20000], [20], 15000, 10, 64, 30),
    Shape("prompt, halves", 4, 28, [3000], [2500], 300, 10, 128, 1),
    Shape("prompt, halves of a longer sequence", 4, 28, [6000], [2500], 300, 10, 128, 1),
    Shape("prompt", 4, 28, [3000], [1200], 300, 10, 256, 1),
    Shape("prompt, splits", 2, 16, [6000] * 4, [512] * 4, 4096, 40, 256, 2),
]
HIDDEN_TREES = [
    Shape("split", 1, 7, [2000], [2], 300, 10, 16, 1),
    Shape("wide", 1, 16, [30000], [16], 17000, 10, 64, 34),
    Shape("prompt, halves, splits", 4, 28, [2500, 300, 333], [200, 190, 200], 1200, 5, 128, 3),
    Shape("prompt, splits", 4, 32, [7000] * 4, [256] * 4, 4500, 70, 256, 2),
]
