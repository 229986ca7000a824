"""The workspace of the residual norm's gradient: no more than its sums."""
from tests.test_residual_cpu import mod  # noqa: F401


def test_four_sums_of_at_most_1024_workgroups(mod):  # noqa: F811
    """Some 512 workgroups, or one for each of at most 1024 gates, with four sums each; for rows that are not held in registers four numbers a row too."""
    lib = mod.load()
    for rows in (1, 7, 513, 1023, 1024, 1025, 4096, 100000):
        for cols in (1, 300, 1000, 4096, 4097, 5000, 8193, 40000):
            for gate in (0, 1, 2, 3, 100, 500, rows):
                n = lib.dmmv_residual_norm_workspace_bytes(rows, cols, gate)
                assert 0 < n <= 1024 * 4 * cols * 4 + 16 * rows + 256, (rows, cols, gate)
                if gate in (0, rows):
                    assert n <= 512 * 4 * cols * 4 + (16 * rows + 256 if cols > 4096 else 0), (rows, cols)
