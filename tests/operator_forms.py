"""Batches that reach the forms of the operators around a projection which small ones do not, shared by the host tests (that they do reach them) and the GPU
tests (what comes out)."""

# (rows, K, N, rank, slots).  The second product takes several pieces of 128 columns in a workgroup from tiles * pieces = 4096 on (2304 above rank 64): two pieces and
# three, widths whose last piece has 64 columns, runs that end early, ranks that are no multiple of 32, both sides of the two LDS buffers (rank 64).
WIDE_FORWARD = [(4100, 64, 7616, 40, 7), (8200, 128, 6208, 24, 5), (4100, 64, 4416, 104, 4), (6001, 64, 3136, 128, 3)]
WIDE_BACKWARD = [(4100, 7616, 64, 40, 7), (8200, 6208, 128, 24, 5), (4100, 4416, 64, 104, 4), (6001, 3136, 64, 128, 3)]
# (rows, depth, rank, slots) whose first product keeps four pieces ahead and asks for more than those (more than 32 pieces of 64)
DEEP = [(1, 4608, 16, 1), (17, 4608, 8, 2), (20, 2176, 32, 3), (33, 3456, 16, 2)]

# (tokens, heads of queries, of keys, head_dim, pairs, rows of positions): several tokens to a workgroup of the forward (from 2048 on), heads that do and do not
# divide its lane groups, one kind alone, a last workgroup with fewer tokens, positions that start again within a workgroup
TOKENS = [(2049, 4, 2, 64, (16, 16), 2049), (3000, 16, 16, 72, (18, 18), 1500), (5003, 1, 3, 72, (10, 20), 7), (9000, 2, 2, 32, (8, 8), 3), (9001, 5, 3, 20, (3, 7), 1),
          (4100, 40, 8, 16, (4,), 1000), (8200, 6, 0, 50, (9, 8, 8), 4100), (6150, 0, 7, 48, (8, 8, 8), 6150), (9000, 1, 1, 2, (1,), 5), (4500, 1, 1, 256, (64, 64), 4)]
