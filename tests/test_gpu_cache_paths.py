"""Attention over a key/value cache on the GPU against the float64 oracle, by the ways in which a launch is cut: each case says which one it
takes, and test_cache_layout.py holds it to that.  Tolerances: test_gpu_cache_attn.py."""

import pytest

from test_gpu_cache_attn import check, make

pytestmark = pytest.mark.gpu


def case(B, H, Hk, Nq, d, P, cap, lens, dtype, decay, q_lens=None, causal=True, grow=0.0, scale=0.0, chunk=None, **layout):
    return dict(B=B, H=H, Hk=Hk, Nq=Nq, d=d, P=P, cap=cap, lens=lens, q_lens=q_lens, causal=causal, dtype=dtype, decay=decay, grow=grow, scale=scale, chunk=chunk,
                layout=layout)


# `chunk`: tiles of an item of own keys.  Lengths are chosen so that many sequences' tiles are no multiple of it
PATHS = {
    # more sequences than a workgroup has threads
    "many_sequences_behind_a_prefix": case(300, 2, 1, 1, 64, 700, 300, [11 * i % 301 for i in range(300)], "bf16", 0.5, chunk=3, pooled=1, joined=1, join_by_row=1, scores_kept=1),
    "many_sequences": case(300, 2, 2, 1, 64, 0, 1100, [37 * i % 1101 for i in range(300)], "fp16", 1.0, chunk=6, pooled=0, joined=1, join_by_row=1, scores_kept=1),
    # more rows to join than one a workgroup
    "rows_joined_behind_a_prefix": case(40, 8, 2, 16, 64, 700, 60, [16 + i for i in range(40)], "bf16", 1.0, q_lens=[i % 17 for i in range(40)], chunk=2, pooled=1, joined=1, join_by_row=0, scores_kept=0),
    "rows_joined": case(20, 16, 2, 20, 128, 0, 900, [97 * i % 901 for i in range(20)], "fp16", 0.9, q_lens=[20 - i % 3 for i in range(20)], chunk=3, many=0, pooled=0, joined=1, join_by_row=0),
    # items of several tiles
    "few_rows": case(16, 4, 4, 1, 128, 0, 7000, [6999 - 371 * i for i in range(16)], "bf16", 1.0, chunk=5, pooled=0, joined=1, scores_kept=1),
    "few_rows_behind_a_long_prefix": case(12, 8, 4, 1, 128, 30000, 700, [700 - 61 * i for i in range(12)], "fp16", 0.3, chunk=4, pooled=1, joined=1, scores_kept=1),
    "prefix_parts_twice_as_long": case(20, 20, 4, 1, 64, 20001, 700, [700 - 35 * i for i in range(20)], "bf16", 1.0, chunk=4, pooled=1, joined=1, scores_kept=1),
    "rows_100": case(6, 40, 2, 5, 128, 0, 9000, [9000, 7777, 5, 6400, 8999, 129], "bf16", 0.5, chunk=4, pooled=0, joined=1, scores_kept=0),
    "pooled_rows_cross_a_tile": case(7, 10, 2, 4, 128, 700, 70, [4, 70, 33, 64, 65, 5, 20], "fp16", 1.0, chunk=1, pooled=1, joined=1, scores_kept=1),
    # the kernel for many queries: its running max raised again and again, in the prefix, in own keys, from part to part, in whole row tiles
    "many_rising_prefix": case(2, 4, 2, 90, 128, 24000, 900, [900, 555], "bf16", 1.0, grow=9.0, scale=0.21, many=1, joined=1),
    "many_rising_prefix_fp16": case(2, 4, 2, 90, 128, 24000, 900, [900, 555], "fp16", 0.0, grow=9.0, scale=0.21, many=1, joined=1),
    "many_rising_own_keys": case(2, 8, 4, 90, 64, 0, 17000, [17000, 12345], "bf16", 1.0, grow=9.0, scale=0.3, many=1, joined=1),
    "many_rising_own_keys_fp16": case(2, 8, 4, 90, 64, 0, 17000, [16999, 64], "fp16", None, q_lens=[90, 33], causal=False, grow=9.0, scale=0.3, many=1, joined=1),
    "many_rising_whole_row_tiles": case(9, 6, 3, 650, 128, 20, 670, [670 - 50 * i for i in range(9)], "bf16", 1.0, q_lens=[max(0, 650 - 90 * i) for i in range(9)], grow=9.0, scale=0.21,
                                        many=1, joined=0, longest_first=1),
    "many_rising_whole_row_tiles_d64": case(12, 8, 4, 700, 64, 0, 700, [700 - 50 * i for i in range(12)], "fp16", 0.5, causal=False, grow=9.0, scale=0.3, many=1, joined=0, longest_first=0),
    # row tiles on all dies in a run: all of them cut, and some
    "many_all_cut": case(9, 6, 3, 650, 128, 20, 4000, [670 - 50 * i for i in range(9)], "bf16", 1.0, causal=False, many=1, joined=1, longest_first=0, row_tiles=162, cut=21, parts=3),
    "many_some_cut": case(20, 8, 8, 257, 128, 0, 4000, [270 + 5 * i for i in range(20)], "fp16", None, causal=False, many=1, joined=1, longest_first=0, row_tiles=320, cut=8, parts=4),
}


@pytest.mark.parametrize("name", PATHS)
def test_against_the_oracle(name):
    c = PATHS[name]
    q, k, v, pk, pv = make(c["B"], c["H"], c["Hk"], c["Nq"], c["d"], c["P"], c["cap"], c["dtype"], 500 + list(PATHS).index(name), grow=c["grow"])
    for b in range(c["B"]):                # what is not in use may hold anything
        k[b, :, c["lens"][b]:] = float("nan")
        v[b, :, c["lens"][b]:] = float("inf")
        if c["q_lens"] is not None:
            q[b, :, c["q_lens"][b]:] = float("nan")
    check(q, k, v, pk, pv, c["lens"], c["q_lens"], c["causal"], c["dtype"], c["decay"], scale=c["scale"], seed=list(PATHS).index(name))
