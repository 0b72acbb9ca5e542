"""Cross-entropy calls that the host sends to the 256 x 256 tiles, with the tile
of each product and what the call covers: (T, d, V, least workspace, slices of
dh: 1, more, or None where a call in pieces chooses).  tests/test_launch_lists_losses_large.py
holds them to their tiles on the CPU; tests/test_gpu_ce_large.py runs them."""

# name: (T, d, V, least, several slices)
CALLS = {
    "one piece, dh in slices": (2049, 512, 16387, 0, True),
    "one piece, dh written directly": (4097, 3840, 2100, 0, False),
    "pieces": (4097, 512, 8200, 1, None),
    "pieces, ragged last one": (5003, 576, 4096 * 2 + 65, 1, None),
}
