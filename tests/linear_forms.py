"""Batches of linear attention by the form that they take on 256 CUs: new tokens, heads, key heads, the blocks of the longest
piece (32 tokens each) and the number of pieces.  tests/test_linear_plan_cpu.py holds the plan to it; the GPU tests run them."""

SHORT, WHOLE, TWO, CUT = "token by token", "whole, a workgroup a head", "whole, two workgroups a head", "in pieces"

# form, tokens, hq, hkv, blocks, pieces: enough blocks for a ring of three or four tiles to go round several times
LONG = {
    "whole": (WHOLE, [400, 391, 413, 385, 416, 399, 410, 401, 5, 70], 64, 16, 13, 9),
    "two": (TWO, [330, 500, 321, 33, 3, 447, 384], 16, 8, 16, 6),
    "pieces": (CUT, [6000], 16, 4, 12, 16),
    "pieces among whole ones": (CUT, [4205, 700, 3, 33], 32, 32, 22, 8),
}

# what the other GPU tests run, by test
SHORTER = {
    "test_equals_the_recurrence": [(SHORT, [1], 32), (SHORT, [2, 0, 5, 1], 4), (TWO, [3, 4, 15, 16, 17], 6), (TWO, [63, 64, 65, 1], 3),
                                   (CUT, [512], 4), (CUT, [1000, 3, 257], 2), (CUT, [2049], 2)],
    "test_a_long_prompt": [(CUT, [8200], 2)],
    "test_whole_chunks_of_many_heads": [(TWO, [200, 64, 129, 31, 200, 96, 200, 7, 200, 200, 161, 33], 64)],
    "test_whole_chunks_few_and_many": [(TWO, [6 + (37 * r) % 91 for r in range(2)], 4), (WHOLE, [6 + (37 * r) % 91 for r in range(70)], 64)],
    "test_states_of_long_whole_chunks": [(WHOLE, [4205, 1494, 2049] * 3 + [4205] * 5, 64), (TWO, [2100, 2049], 64), (TWO, [1494, 1400], 64)],
}
