"""Which kernels the norm's, the activation's and the few tokens' calls launch, and how much LDS they ask for, without a GPU."""
import pytest

import launch_recorder


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    return launch_recorder.build(tmp_path_factory.mktemp("launches"))


def test_kernels_of_a_few_tokens(recorder):
    """Two launches where up to four tokens choose inside the first, with activations in LDS; elsewhere one for the choice, and one more for
    the sum over a token's experts; never more LDS than is granted."""
    result = launch_recorder.run(recorder, r"""
result = []
for T, E, K, H, F, groups, bias, here, out in ((1, 128, 8, 2048, 768, 1, 0, 128, 0), (1, 32, 8, 7168, 2048, 1, 1, 32, 0), (4, 256, 8, 7168, 2048, 8, 1, 32, 0),
        (4, 16, 16, 512, 128, 1, 0, 16, 1), (5, 16, 8, 512, 128, 1, 0, 16, 0), (1, 12, 2, 512, 128, 3, 0, 12, 0), (1, 2000, 8, 512, 128, 1, 0, 512, 0),
        (1, 40, 20, 512, 128, 1, 0, 40, 0), (1, 8, 2, 512, 128, 1, 1, 8, 0), (20, 8, 2, 512, 128, 1, 0, 8, 0), (64, 8, 2, 512, 128, 1, 0, 8, 1),
        (64, 256, 8, 7168, 2048, 8, 0, 32, 0), (19, 60, 6, 1030, 1001, 1, 0, 60, 1), (64, 64, 1, 256, 128, 1, 0, 64, 0), (8, 64, 8, 256, 1 << 19, 1, 0, 2, 0),
        (64, 1024, 16, 128, 128, 1, 0, 1024, 0)):
    r = ctypes.byref(B.hm_router(E, K, 1 if bias else 0, groups, 1, 1, 1, 1.0))
    rc = L.hm_layer_few(at(1), H, at(2), 1, E, at(3) if bias else None, T, r, at(4), at(5), at(6), at(7), 0, here, H, F, at(8), at(9), at(10), out, at(11), 1 << 40, None)
    result.append([[T, E, K, H, F, groups, here, out], rc, launched()])
""")
    for (T, E, K, H, F, groups, here, out), rc, launches in result:
        names = [k["name"].split("<")[0] for k in launches]
        assert rc == 0, (T, E, K, H, F)
        inside = T <= 4 and K <= 16 and groups in (1, 2, 4, 8, 16) and E <= 1024
        staged = 2 * (2 + out) * T * K * ((F + 127) // 128 * 128 + 8) + 8 * T * 16 * 4
        few = T * K <= 64 and staged <= 66 * 1024
        chosen = [] if inside else ["route_lists_kernel" if K <= 16 and groups != 3 and E <= 1024 else "route_kernel"]
        assert names == chosen + ["few_up_kernel"] + (["few_down_kernel"] if few else ["few_down_slots_kernel", "few_sum_kernel"]), (T, E, K, H, F, names)
        for k in launches:
            assert k["lds"] <= k["granted"], k
        if few:
            assert launches[-1]["lds"] == staged and launches[-1]["grid"][0] == -(-H // (8 if H < 4096 else 16))
        up = launches[len(chosen)]
        assert up["grid"][:2] == [(F + 127) // 128 * 8, min(here, T * K)] and up["block"][0] == 256
        if not inside:   # how many slots a workgroup takes at a time
            assert up["name"].split(",")[2].strip() == ("1" if T <= 16 or T * K <= 10 * E else "4"), up["name"]


def test_kernels_of_the_norm_hold_a_row(recorder):
    """Threads times vectors times eight values are no less than the row, whatever its length and the number of rows, and a launch has all
    groups; the way back adds up its parts where there are more than one."""
    result = launch_recorder.run(recorder, r"""
result = []
for rows in (1, 2, 256, 257, 1000, 100000, 1 << 31):
    for C in list(range(1, 40)) + [500, 511, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097, 7168, 8192, 8193, 16384, 16385, 32768]:
        for dtype, total in ((0, 0), (0, 1), (1, 1), (1, 0)):
            rc = L.hm_rms_norm(at(1), dtype, C, at(2), total, C, at(3), 1, 1e-6, min(rows, (1 << 31) - 1), C, at(4), C, at(5), 0, at(6), at(7), None)
            a = launched()
            rb = L.hm_rms_norm_backward(at(1), dtype, C, at(2), total, C, at(3), 1, 1e-6, min(rows, (1 << 31) - 1), C, None, 0, at(4), C, at(5), at(6), 1 << 40, None)
            result.append([rows, C, rc, rb, a, launched(), L.hm_rms_norm_backward_workspace_bytes(min(rows, (1 << 31) - 1), C)])
""")
    shape = lambda name: [int(v) for v in name[name.index("<") + 1:-1].split(",")[-2:]]
    for rows, C, rc, rb, forward, backward, bytes_ in result:
        assert rc == rb == 0 and len(forward) == 1
        vectors, threads = shape(forward[0]["name"])
        assert vectors * threads * 8 >= C and forward[0]["block"][0] == max(threads, 256)
        assert vectors * threads * 8 < 2 * C or C <= (1024 if rows <= 512 else 512)   # most have something to do
        assert forward[0]["grid"][0] <= 2048
        vectors, threads = shape(backward[0]["name"])
        groups = min(rows, 1024 if C <= 1024 else 512)
        assert vectors * threads * 8 >= C and backward[0]["grid"][0] * max(256 // threads, 1) >= groups > (backward[0]["grid"][0] - 1) * max(256 // threads, 1)
        assert len(backward) == (1 if groups == 1 else 2) and bytes_ == (0 if groups == 1 else 4 * C * groups)


def test_kernels_of_the_activation(recorder):
    """Columns in 8 bits come from the tiles, and rows too where both halves are whole blocks; without columns everything is by rows."""
    result = launch_recorder.run(recorder, r"""
result = []
for dtype in (0, 1):
    for rows, F, S in ((1, 1, 1), (300, 128, 2), (300, 130, 2), (40000, 768, 16), (100, 1 << 19, 1)):
        for gh, q, qc, ac in ((1, 0, 0, 0), (0, 1, 0, 0), (1, 1, 1, 1), (0, 1, 1, 0), (0, 0, 0, 1), (1, 0, 1, 0)):
            p = lambda i, on: at(i) if on else None
            rc = L.hm_gated_backward(at(1), at(2), dtype, 2 * F, F, at(3), S, rows, F, p(4, gh), 0, p(5, q), p(6, q), p(7, qc), p(8, qc), p(9, ac), p(10, ac), None)
            result.append([dtype, rows, F, S, gh, q, qc, ac, rc, launched()])
""")
    for dtype, rows, F, S, gh, q, qc, ac, rc, launches in result:
        names = [k["name"].split("<")[0] for k in launches]
        assert rc == 0
        by_tiles = bool(qc or ac)
        by_rows = not by_tiles or (q and F % 128 != 0)
        assert names == ["gated_backward_kernel"] * by_tiles + ["gated_backward_rows_kernel"] * by_rows, (rows, F, names)
        if by_tiles:
            tiles = -(-(rows // 128 + S) * -(-F // 128) // 8) * 8
            assert launches[0]["grid"][0] == min(tiles, 256) and launches[0]["name"].endswith("true>" if gh else "false>")
        if by_rows:
            assert launches[-1]["grid"][0] == -(-rows * -(-2 * F // 512) // 4)


def test_few_tokens_of_a_router_of_many_groups(recorder):
    """More groups than the 16 lanes that choose inside the first product: hm_route's kernel makes the choice, as it does alone."""
    result = launch_recorder.run(recorder, r"""
result = []
for E, groups in ((272, 17), (320, 20), (256, 32), (64, 64), (4096, 4096)):
    for T in (1, 4, 5, 64):
        for logits in (0, 1):
            r = ctypes.byref(B.hm_router(E, 4, 1, groups, 4, 1, 1, 1.0))
            rc = L.hm_route(at(2), logits, E, at(3), T, r, at(8), at(9), None)
            alone = launched()
            few = L.hm_layer_few(at(1), 512, at(2), logits, E, at(3), T, r, at(4), at(5), at(6), at(7), 0, 8, 512, 128, at(8), at(9), at(10), 0, at(11), 1 << 40, None)
            result.append([E, groups, T, rc, few, alone, launched()])
""")
    for E, groups, T, rc, few, alone, launches in result:
        assert rc == few == 0, (E, groups, T)
        assert alone[0]["name"].startswith("route_kernel") and launches[0] == alone[0]
        assert [k["name"].split("<")[0] for k in launches[1:]] == ["few_up_kernel"] + (["few_down_kernel"] if T <= 5 else ["few_down_slots_kernel", "few_sum_kernel"])


def test_lds_is_granted_on_every_device(recorder):
    """What a kernel may have beyond the default is a device's: a second device of the process is asked too, once."""
    result = launch_recorder.run(recorder, r"""
result = []
r = ctypes.byref(B.hm_router(32, 8, 1, 1, 1, 1, 1, 1.0))
for device in (0, 1, 0, 3, 1):
    recorder.recorder_device(device)
    for out in (0, 1):
        rc = L.hm_layer_few(at(1), 7168, at(2), 1, 32, at(3), 1, r, at(4), at(5), at(6), at(7), 0, 32, 7168, 2048 >> out, at(8), at(9), at(10), out, at(11), 1 << 40, None)
        result.append([device, rc, launched()])
""")
    for device, rc, launches in result:
        assert rc == 0 and launches[-1]["name"].startswith("few_down_kernel")
        assert launches[-1]["lds"] <= launches[-1]["granted"], (device, launches[-1])
