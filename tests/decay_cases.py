"""Prompts of linear attention whose runs' sums a launch of its own adds up (k_decay_join): more than two groups of eight
runs, of two chunks and more, in one sequence; sequences that begin behind such a group's end; more sequences than a wave
has lanes.  (new tokens, held, heads, key heads, head_dim, rows behind the last sequence); test_decay_plan.py holds the plan
to them."""
JOINED = [([5000], [1], 2, 1, 128, 3), ([5003], [0], 1, 1, 128, 0), ([7001], [1], 2, 2, 64, 3),
          ([700, 5000], [1, 0], 3, 3, 128, 3), ([5000, 700], [1, 1], 3, 1, 128, 3),
          ([300, 5200, 0, 64], [0, 1, 1, 1], 2, 1, 128, 3), ([40, 7000], [1, 1], 3, 1, 64, 3),
          ([1100, 9000], [1, 1], 1, 1, 64, 3), ([3] * 70 + [6000], [0, 1] * 35 + [1], 1, 1, 128, 3)]
# bounds far above the lengths: the same launch over fewer runs than planned
PADDED = [([2900], [1], 2, 1, 128, 2500), ([100, 3000], [1, 1], 1, 1, 64, 4000)]
# as they are in the test of calls that agree bit for bit: three heads, one key head
AGREE = [([5000], 128), ([7000, 40], 64), ([700, 5000], 128)]
