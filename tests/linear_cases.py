"""Layers that reach every form of hb_linear_q4's kernel: (form, rows, inputs, outputs).  Inputs odd and over several rounds of a workgroup's steps (one round is
4096 inputs in forms 0 and 8, 2048 in 1 to 3, 1024 in 4, 512 in 5, 256 in 6 and 7), a last tile of rows that is not full, a part of a tile of outputs."""
EVERY_FORM = [(0, 3, 9001, 33), (0, 1, 1001, 70), (1, 259, 4301, 5), (2, 5, 4301, 2117), (3, 9, 4301, 2050), (4, 13, 2301, 3001), (4, 259, 1301, 67),
              (5, 343, 1301, 131), (5, 29, 801, 4101), (6, 227, 1301, 2061), (7, 19, 1301, 20011), (8, 1, 9001, 16401)]
GROUPS = [32, 64, 128]                     # each is a kernel of its own; in groups of 32 form 3 stands in for form 8


def cases():
    for group in GROUPS:
        for form, *sizes in EVERY_FORM:
            yield (3 if form == 8 and group == 32 else form, *sizes, group)
