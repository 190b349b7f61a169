"""Products of an expert layer that take tiles of 256 x 256, more than the card has CUs: a workgroup has two of them or more.  Shared by
test_moe_choice.py (that they do) and test_gpu_moe_wide.py (what comes out).  E 0: no routing; dropped: a share of the entries."""

# T, k, E, d_in, d_out, activation, dropped: rows and columns that end inside a tile, inputs that end inside a step
FORWARD = [(3700, 1, 0, 328, 7640, "none", 0.0), (4000, 1, 0, 456, 8120, "gelu", 0.0), (4000, 1, 0, 328, 4040, "swiglu", 0.0),
           (2050, 2, 3, 520, 6640, "none", 0.1), (4100, 1, 2, 776, 7112, "silu", 0.2), (2000, 2, 4, 904, 3400, "swiglu", 0.1)]
# the inputs are the columns here, the outputs are summed over; the activation before the product
DX = [(3700, 1, 0, 7640, 328, "none", 0.0), (2050, 2, 3, 6640, 584, "gelu", 0.1), (4100, 1, 2, 7112, 776, "swiglu", 0.2)]
# one matrix; uneven experts, which are ranked and take every other turn backwards; more experts than are ranked
DW = [(300, 1, 0, 8184, 4072, 0.0), (9000, 2, 16, 2024, 1992, 0.1), (74000, 2, 144, 1000, 1016, 0.05)]


def tiles(rows, cols):
    return -(-rows // 256) * -(-cols // 256)


def columns(d_out, activation):
    """of y, twice as many as a tile takes where gates and what goes with them lie side by side"""
    return 2 * d_out if activation == "swiglu" else d_out
# through a z kept in 8 bits: several activations of a shape; a second half of swiglu's that begins inside a block of 32 columns
DX_KEPT = [(3700, 1, 0, 7640, 328, ("relu", "swiglu"), 0.0), (2050, 2, 3, 6640, 584, ("gelu", "silu"), 0.1), (4100, 1, 2, 7112, 776, ("swiglu", "silu"), 0.2)]
# 8-bit integers, of which a step takes 128 of r: inputs that end inside a step, experts whose last tiles are ragged, rows of no expert between them
INT8 = [(3700, 1, 0, 656, 7640, "none", 0.0), (4000, 1, 0, 912, 8120, "gelu", 0.0), (4000, 1, 0, 656, 4040, "swiglu", 0.0),
        (2050, 2, 3, 528, 6640, "relu", 0.1), (4100, 1, 2, 1552, 7112, "silu", 0.2), (2000, 2, 4, 1040, 3400, "swiglu", 0.1)]
