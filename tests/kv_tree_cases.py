"""Calls of ls_kv_attention_tree that reach the parts of its kernel that depend on how the
work is divided, and what they are there for.  `reaches`: rows of a tile; the least number of
pieces that some head falls into (above 16 they are joined in groups); the least number of steps in
some piece (pages are looked up 32 steps at a time), 128 tokens each.  cus: compute units that the
context is told to use (0: the device's 256).  width: tokens that a row of the page table covers at least."""


def case(D, seqs, reaches, H=1, G=4, cus=0, width=0, window=0, sinks=0, absent=()):
    return dict(D=D, seqs=seqs, reaches=reaches, H=H, G=G, cus=cus, width=width, window=window, sinks=sinks, absent=absent)


def cases():
    out = {}
    for D in (64, 128, 256):
        # one long sequence: pieces in groups, 32 rows to a tile
        out[f"groups {D}"] = case(D, [(60000, 5)], (32, 33, 1))
        out[f"groups {D} of two heads"] = case(D, [(1, 1), (60001, 3), (33, 4)], (32, 17, 1), H=2)
        # few compute units: long pieces, whose pages are looked up more than once; some pages are not there
        out[f"long pieces {D}"] = case(D, [(20000, 5)], (32, 2, 65), cus=1, absent=[(0, j) for j in range(560, 700, 3)])
        out[f"long pieces {D}, window"] = case(D, [(15000, 5), (300, 8)], (32, 2, 33), cus=2, window=12345, sinks=20)
    for D in (64, 128):
        # 64 rows to a tile, by rows and the table's width: cut heads, in groups of pieces and in long ones
        out[f"tall {D}"] = case(D, [(20000, 64)], (64, 9, 1), H=2, width=1 << 18)
        out[f"tall groups {D}"] = case(D, [(60000, 64)], (64, 33, 1), width=1 << 18)
        out[f"tall long pieces {D}"] = case(D, [(20000, 64)], (64, 4, 33), width=1 << 18, cus=8, absent=[(0, j) for j in range(300, 400, 3)])
        out[f"tall whole heads {D}"] = case(D, [(9000, 64)], (64, 1, 65), width=1 << 18, cus=1)
        # 64 rows to a tile, by the number of tiles
        out[f"tall by tiles {D}"] = case(D, [(20000, 8)] + [(40 + b, 8) for b in range(7)], (64, 2, 1), H=2, G=8, cus=8)
    return out
