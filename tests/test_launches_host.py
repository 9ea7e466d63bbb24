"""What the operators around the loss pass launch and prepare, seen from the host."""

from launch_recorder import recorded


def test_one_product_of_any_size_prepares_all_its_kernels(tmp_path):
    """A kernel that needs an attribute has it after the first call, so that a later call of another size can be captured."""
    got = recorded(tmp_path, """
        lib.fopd_mx4_bytes.restype = lib.fopd_mx4_logits_workspace_bytes.restype = c_size_t
        lib.fopd_mx4_bytes.argtypes, lib.fopd_mx4_logits_workspace_bytes.argtypes = 2 * [c_int64], 3 * [c_int64]
        lib.fopd_mx4_logits.argtypes = [P, c_int, c_int64, P, c_size_t, c_int64, c_int64, c_int64, P, c_int, c_int64, P, c_size_t, P]
        result = []
        # (rows, vocabulary, width, type): few, some and many rows, tiles that walk and tiles that do not, of both types
        for T, V, d, dt in ((1, 1000, 64, 1), (45, 1000, 64, 1), (100, 40000, 64, 0), (300, 30000, 256, 1), (300, 30000, 256, 0),
                            (4096, 32000, 1024, 1), (4096, 32000, 1024, 0), (4096, 32000, 16777216, 0)):
            st = lib.fopd_mx4_logits(P(4096), 1, (d + 7) // 8 * 8, P(4096), lib.fopd_mx4_bytes(V, d), T, V, d, P(4096), dt, V,
                                     P(4096), lib.fopd_mx4_logits_workspace_bytes(T, V, d), None)
            result.append((st, count("launches"), count("attribute_calls")))
        kernels = (P * count("launches")).in_dll(rec, "launched")
        result.append(len(set(kernels)))
    """)
    *calls, kernels = got
    assert all(st == 0 for st, _, _ in calls)
    assert [n for _, n, _ in calls] == sorted({n for _, n, _ in calls})      # each launched something
    assert calls[0][2] > 0 and all(n == calls[0][2] for _, _, n in calls), calls
    assert kernels == 8                                      # (packing, few rows as they are and packed, some rows, all four of tiles)
