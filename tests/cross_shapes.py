"""Sizes of attention to an encoder's states that reach what the host's rules choose, for the GPU's tests and those of
the rules: (B, N, S, H, Hkv, D)."""

# Parts of the states joined by a row's lanes: every width that rows are padded to, exactly and not; two to
# sixteen parts.
FEW_PARTS = [(3, 6000, 300, 1, 1, 16), (1, 9000, 300, 1, 1, 32), (2, 2100, 2500, 2, 1, 32), (3, 1500, 2500, 1, 1, 48), (1, 4500, 700, 1, 1, 64),
             (1, 2100, 700, 1, 1, 80), (3, 800, 1500, 1, 1, 128)]
# All states in LDS, in both directions (float32: 16 wide alone).
WHOLE = [(4, 33_000, 66, 4, 4, 32), (1, 140_000, 70, 4, 4, 64), (2, 70_000, 70, 4, 4, 64), (1, 140_000, 40, 4, 1, 48), (4, 66_000, 67, 4, 2, 16)]
# The most states that LDS holds, by type and width, with enough rows.
LDS_STATES = {("bf16", 16): 2496, ("bf16", 32): 1216, ("bf16", 64): 576, ("fp32", 16): 832}
LDS_ROWS = (1, 140_000, 4, 4)  # B, N, H, Hkv
# Many samples and shared heads: of a few rows, and of enough for workgroups of four blocks a wave, but one round of them
# and a bit (both in the four-wave kernels), or two rounds and nearly one (all states in LDS).
MANY = [(1500, 70, 50, 4, 4, 32), (4500, 1, 20, 4, 4, 16), (33, 1050, 33, 16, 8, 16), (64, 2100, 40, 8, 8, 32), (30, 1100, 33, 16, 8, 16)]


def some_lengths(B, S):
    """The first sample's states all there (of a single one: a third), then none, one and every other part."""
    return [S // 3 if B == 1 else S] + [(0, 1, S // 2)[b % 3] for b in range(B - 1)]
