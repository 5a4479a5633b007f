"""Products that go to the large tiles, for the tests of their results on the GPU and of the rule that sends them there.

A product is named by what it is in terms of its three sizes (m, n outer, k contracted) and by which operands lie across: "forward" none,
"da" the second, "db" both.  pad: elements behind a row, so that rows are whole vectors whatever their length.  tile, half: what the rule
gives; half tiles are those 256 x 128 ones that whole rounds of 256 x 256 leave, in a launch of their own."""
import torch

BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn

# kind, dtype, m, n, k, tile, half.  9 whole steps and more, so that the schedule of a step with two to follow runs several times and the
# XCDs begin at different steps; contractions that end inside a step; results that end inside a tile, in rows and in columns.
LARGE = [
    ("forward", BF16, 4096, 4096, 600, 256, 0),
    ("forward", BF16, 4091, 4085, 603, 256, 0),
    ("forward", BF16, 4093, 4611, 603, 256, 3),
    ("forward", BF16, 4096, 4608, 640, 256, 2),
    ("forward", E4M3, 4096, 4096, 1200, 256, 0),
    ("forward", E4M3, 4091, 4085, 1203, 256, 0),
    ("forward", E4M3, 4093, 4611, 1203, 256, 3),
    ("forward", E4M3, 4096, 4608, 2304, 256, 2),
    ("da", BF16, 4091, 4088, 603, 256, 0),
    ("da", BF16, 4096, 4096, 1152, 256, 0),
    ("da", BF16, 4093, 4616, 603, 256, 3),
    ("db", BF16, 4088, 4080, 603, 256, 0),
    ("db", BF16, 4096, 4096, 1152, 256, 0),
    ("db", BF16, 4088, 4616, 603, 256, 3),
]

# The same of smaller tiles, in one part and in several, with steps enough for their schedules.
SMALLER = [
    ("forward", BF16, 2000, 2000, 1203, 128, 0),
    ("forward", E4M3, 2000, 2000, 2403, 128, 0),
    ("forward", BF16, 200, 520, 4099, 128, 0),
    ("forward", BF16, 64, 14336, 1203, 64, 0),
    ("forward", E4M3, 61, 14336, 2403, 64, 0),
    ("forward", BF16, 40, 1000, 4163, 64, 0),
    ("da", BF16, 2000, 2000, 1203, 128, 0),
    ("da", BF16, 200, 520, 4099, 128, 0),
    ("db", BF16, 2000, 2000, 1203, 128, 0),
    ("db", BF16, 200, 520, 4099, 128, 0),
]


def pad_to_vectors(length, dtype):
    return -length % (16 // torch.empty(0, dtype=dtype).element_size())
