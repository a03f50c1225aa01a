"""Products with an epilogue that the tile choice gives to each kernel, at 256 compute units.

The small shapes cannot be forced, so a product stands for each; test_activation_calls.py checks on the host that it
still gets its kernel, test_gpu_activation.py that the kernel computes it.  n counts outputs: a gated product has
twice as many operand rows.
"""
# kernel name part (after the formats), gated, m, n, k
TILES = [
    ("act_ring_kernelILb0ELi0ELi0ELi64ELi64ELi4E", False, 65, 62, 600),
    ("act_ring_kernelILb1ELi0ELi0ELi64ELi64ELi4E", True, 65, 62, 600),
    ("act_ring_kernelILb0ELi0ELi0ELi128ELi64ELi3E", False, 8862, 386, 600),
    ("act_ring_kernelILb1ELi0ELi0ELi128ELi64ELi3E", True, 8862, 193, 600),
    ("act_ring_kernelILb0ELi0ELi0ELi128ELi64ELi6E", False, 68, 8257, 1000),
    ("act_ring_kernelILb1ELi0ELi0ELi128ELi64ELi6E", True, 68, 4130, 1000),
    ("act_ring_kernelILb0ELi0ELi0ELi64ELi128ELi3E", False, 129, 27693, 300),
    ("act_ring_kernelILb1ELi0ELi0ELi64ELi128ELi3E", True, 129, 13846, 300),
    ("act_ring_kernelILb0ELi0ELi0ELi64ELi128ELi6E", False, 33, 16407, 900),
    ("act_ring_kernelILb1ELi0ELi0ELi64ELi128ELi6E", True, 33, 8203, 900),
    ("act_ring_kernelILb0ELi0ELi0ELi128ELi128ELi2E", False, 198, 26498, 400),
    ("act_ring_kernelILb1ELi0ELi0ELi128ELi128ELi2E", True, 198, 13249, 400),
    ("act_ring_kernelILb0ELi0ELi0ELi128ELi128ELi4E", False, 65, 25277, 700),
    ("act_ring_kernelILb1ELi0ELi0ELi128ELi128ELi4E", True, 65, 12638, 700),
]
# the large shapes can be forced: qe.TILE_256x256, qe.TILE_192x256
