"""Sizes (N, C, F, tile) of the gated feed-forward's tests that are long enough for its kernels' loops
to turn over: rings of LDS slots used several times, registers that rotate, tiles that add to the
sums of the ones before.  test_gated_rules.py holds what they reach, by the library's own rules."""

# Forward and backward.
LONG = [(34_001, 64, 300, 17_000), (34_001, 128, 480, 17_000), (34_001, 128, 290, 17_000), (34_001, 128, 340, 17_000),
        (34_001, 192, 288, 17_000), (34_001, 256, 320, 17_000), (34_001, 256, 256, 17_000), (4097, 176, 700, 3000),
        (4097, 256, 700, 3000)]
# Forward, also in place: calls of about a workgroup per compute unit.
MIDDLE = [(20_001, C, F) for C in (48, 128, 192, 256) for F in (100, 150)] + [(4097, 64, 700), (4097, 112, 700)]
