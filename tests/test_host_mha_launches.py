"""CPU checks of how attention with row sums is launched, on the stand-in runtime."""

from test_host_launches import libs, run  # noqa: F401

CALLS = r"""
def forward(nq, nk, heads, kv, d, seqs=1, dtype=A.ACID_BF16):
    b = p[10] if seqs > 1 else None
    m = A.acid_mha(nq=nq, nk=nk, dtype=dtype, heads=heads, kv_heads=kv, head_dim=d, scale=1.0, sequences=seqs, q_bounds=b,
                   k_bounds=b, frame_rows=0, frames_before=-1, frames_after=-1, q_first=0)
    fk.launches = 0
    assert lib.acid_mha_forward(C.byref(m), p[0], heads * d, p[1], kv * d, p[2], kv * d, p[3], heads * d, p[4], p[5], 1 << 40,
                                None) == A.ACID_OK, lib.acid_last_error()
    return fk.launches, fk.grid
"""


def test_a_few_rows_go_to_their_kernel_while_that_is_the_faster_one(libs):  # noqa: F811
    """The last launch is the join of a row's shares, a CTA to a row and head; on tiles it is the merge of split tiles, a
    CTA to eight rows of 256, or one kernel on all 152 SMs."""
    run(CALLS + """
F = A.ACID_FP32
few = [((1, 32760, 12, 12, 128), 12), ((1, 32760, 16, 1, 128), 16), ((1, 5000, 24, 8, 128), 24), ((4, 512, 12, 12, 128), 48),
       ((2, 4726, 12, 12, 128), 24), ((4, 4726, 4, 4, 64, 1, F), 16), ((2, 2 * 4096, 12, 12, 128, 2), 24),
       ((16, 8 * 512, 8, 1, 64, 8), 128), ((2, 32760, 24, 8, 128), 48)]
for args, rows in few:
    assert forward(*args) == (2, rows), (args, fk.launches, fk.grid)
# two to four rows whose products with the keys are many, evenly or in one of the sequences
for args in ((4, 32760, 12, 12, 128), (3, 32760, 24, 8, 128), (4, 32760, 16, 1, 128), (4, 32760, 30, 30, 64)):
    launches, grid = forward(*args)
    assert (launches, grid) == (2, args[2] * 256 // 8), (args, launches, grid)
for args in ((253, 65 * 1000, 12, 12, 128, 64), (256, 64 * 512, 24, 8, 128, 64), (128, 64 * 4096, 12, 12, 128, 64)):
    assert forward(*args) == (1, 152), (args, fk.launches, fk.grid)
""", *libs)
