"""Sizes (groups, tokens, vocabulary, columns) at which the vocabulary loss and its gradient are cut in the ways that the tests have to reach; what
each is for is checked against the plan without a GPU."""

# gradient: several tiles of dW a task (run_w), the last task with fewer; dH's contraction in parts
RUNS_OF_DW = [(32, 64, 30000, 128), (40, 100, 4700, 72), (3, 40, 69800, 520)]
# gradient: several pieces of the vocabulary, dH in parts, several tiles along the columns
PIECES = [(3, 2100, 17000, 300), (2, 1500, 50000, 520)]
# ... of sums that are cut, of 16-bit types
LONG = [(2, 8300, 9000, 600), (1, 70, 5000, 8264)]
# loss: several tiles a task, each in several sums
RUNS_OF_LOSS = [(2, 2100, 20000, 1000), (1, 3000, 60000, 1100)]
# loss of one or two tokens a group: just below and above what the form of few tokens takes of 16-bit types
FEW, NOT_FEW = [(1, 1, 1 << 17, 72), (4, 2, 1 << 14, 256)], [(1, 1, (1 << 17) + 1, 72), (4, 2, 100000, 256), (64, 1, 5000, 300)]
