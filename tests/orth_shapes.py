"""Lists of matrices that reach the products by tiles of 128, for the GPU's tests and those of the host's rules."""

# K of two to eight steps and tiles half of padding, one a workgroup and several; rounds of them with ragged ends, wide,
# tall and batches; X X^T of long rows.
STREAM = [[(64, 128)] * 100 + [(128, 64)] * 60 + [(40, 50, 120)], [(64, 128)] * 1100, [(256, 1000)] * 40 + [(900, 250)] * 40,
          [(1003, 1500), (1500, 1003)] * 2]
# Of each list, whether its symmetric products and its updates take tiles of 128.
REACHED = [(True, True), (True, True), (True, True), (True, False)]
