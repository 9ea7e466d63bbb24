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


def test_scaling_goes_through_the_list_from_its_end(tmp_path):
    """fopd_grad_norm reads the tensors in order and leaves the last ones in the cache; fopd_grad_scale takes a table's pieces from
    the last one down, so tables hold the list's order and come from its end."""
    got = recorded(tmp_path, """
        class Entry(Structure):
            _fields_ = [("grad", c_int64), ("out", c_int64), ("cols", c_int64), ("ld", c_int64), ("ld_out", c_int64), ("rows", c_int32),
                        ("row_pieces", c_int32), ("first_piece", c_int32), ("bf16", c_int8), ("out_bf16", c_int8)]
        class Table(Structure):
            _fields_ = [("n", c_int32), ("pieces", c_int32), ("t", Entry * 48)]
        class Tensor(Structure):
            _fields_ = [("grad", c_int64), ("out", c_int64), ("rows", c_int64), ("cols", c_int64), ("ld", c_int64), ("ld_out", c_int64),
                        ("dt", c_int), ("dt_out", c_int)]
        lib.fopd_grad_norm.argtypes = [P, c_int32, c_int, P, P, P, c_size_t, P]
        lib.fopd_grad_clip.argtypes = [P, c_int32, P, c_float, c_float, P, P]
        c_int.in_dll(rec, "argument_bytes").value = sizeof(Table)
        result = []
        for n in (1, 2, 41, 48, 49, 130):
            # one piece, several, rows with gaps and nothing at all, at addresses that count up
            shapes = [[(3, 5, 5), (1, 30000, 30000), (7, 100, 104), (0, 5, 5)][(i + 1) % 4] for i in range(n)]
            ts = (Tensor * n)(*[Tensor(1 << 20 | i << 8, 1 << 20 | i << 8, r, c, ld, ld, i % 2, i % 2) for i, (r, c, ld) in enumerate(shapes)])
            begin = count("launches")
            assert lib.fopd_grad_norm(ts, n, 0, P(4096), None, P(4096), 1 << 20, None) == 0
            middle = count("launches")
            assert lib.fopd_grad_clip(ts, n, P(4096), 1.0, 0.0, None, None) == 0
            raw = (c_char * 4096 * count("launches")).in_dll(rec, "arguments")
            tables = [Table.from_buffer_copy(raw[k][:sizeof(Table)].ljust(sizeof(Table), bytes(1))) for k in range(begin, count("launches"))]
            told = [[g.pieces, [[e.grad >> 8 & 4095, e.first_piece, e.rows * e.row_pieces] for e in g.t[:g.n]]] for g in tables]
            result.append([n, told[:middle - begin], told[middle - begin:]])
    """)
    for n, norm, scale in got:
        present = [i for i in range(n) if (i + 1) % 4 != 3]
        for pieces, entries in norm + scale:
            at = 0
            for _, first, count in entries:
                assert first == at
                at += count
            assert at == pieces
        assert [e[0] for _, entries in norm for e in entries] == present
        assert len(scale) == (len(present) + 47) // 48
        assert [e[0] for _, entries in reversed(scale) for e in entries] == present, (n, scale)


def test_products_take_the_kernel_that_measured_fastest(tmp_path):
    """Either side of each border between the kernels of few rows, of some and of tiles, told from each other by their workgroups."""
    cases = {"few": [(49, 32000), (64, 32768), (96, 16384), (128, 16384), (129, 21504), (160, 21824), (161, 21824), (192, 21824), (256, 16384), (256, 22528),
                     (512, 11264), (1024, 4352), (1024, 5632), (4096, 1024)],
             "stream": [(49, 32769), (64, 40000), (65, 16385), (96, 24000), (128, 24000), (129, 21889), (160, 24000), (160, 151936)],
             "tiles": [(161, 21889), (192, 27264), (192, 25600), (256, 17600), (256, 22592), (448, 11648), (512, 13568), (1024, 4800), (1024, 5888), (4096, 151936)]}
    got = recorded(tmp_path, """
        lib.fopd_mx4_bytes.restype = lib.fopd_mx4_logits_workspace_bytes.restype = c_size_t
        lib.fopd_mx4_bytes.argtypes, lib.fopd_mx4_logits_workspace_bytes.argtypes = 2 * [c_int64], 3 * [c_int64]
        lib.fopd_mx4_logits.argtypes = [P, c_int, c_int64, P, c_size_t, c_int64, c_int64, c_int64, P, c_int, c_int64, P, c_size_t, P]
        result = {}
        for name, sizes in CASES.items():
            for T, V in sizes:
                before, d = count("launches"), 4096
                assert lib.fopd_mx4_logits(P(4096), 1, d, P(4096), lib.fopd_mx4_bytes(V, d), T, V, d, P(4096), 1, (V + 7) // 8 * 8, P(4096),
                                           lib.fopd_mx4_logits_workspace_bytes(T, V, d), None) == 0
                assert count("launches") == before + 2                     # the rows' packing, then the product
                grid = (c_uint * count("launches")).in_dll(rec, "grids")[before + 1]
                kind = {(V + 63) // 64: "few", (V + 127) // 128: "stream"}.get(grid, "tiles")
                result["%s %d %d" % (name, T, V)] = kind
    """.replace("CASES", repr(cases)))
    assert len(got) == sum(map(len, cases.values()))
    assert not {k: v for k, v in got.items() if k.split()[0] != v}
