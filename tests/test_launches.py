"""What is launched, looked at on the host: where kernels read in LDS, how much of it a launch asks for, and which kernel a call
takes, for calls whose results would not show it."""
import os
import subprocess

import pytest

import launch_recorder

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    return launch_recorder.build(tmp_path_factory.mktemp("launches"))


def test_products_of_the_swap_tables_stay_inside_their_tiles(tmp_path):
    """Every tile that a wave of swap_cooc_kernel multiplies lies in the rows that its launch asks LDS for, for all experts and
    groups, also where another cut has fewer groups than the one the launch is sized for."""
    (tmp_path / "walk.cpp").write_text(r"""
#include <cstdio>
#include "hm_cooc.h"
template <int COLS> static int walk(int E, int ng) {
  typedef hm::CoocTiles<COLS> layout;
  const layout t(E, ng);
  int bad = t.rows() != 32 * ((E + 31) / 32 + COLS + (ng + 31) / 32), c = 0, g = 0;
  auto inside = [&](int first, int tiles, int from, int to) { return first >= from && first + 32 * tiles <= to; };
  for (int w = 0; w < hm::kCoocWaves; ++w) {
    if (t.has_c(w)) ++c, bad += !inside(t.c_rows(w), 1, 0, t.s_at()) + !inside(t.c_columns(w), layout::kColumnsOfC, t.s_at(), t.m_at());
    if (t.has_g(w)) ++g, bad += !inside(t.g_rows(w), 1, t.s_at(), t.m_at()) + !inside(t.g_columns(w), layout::kColumnsOfG, t.m_at(), t.rows());
    if (COLS > 1) bad += t.has_c(w) && t.has_g(w);   // these share their sums
  }
  bad += c != (E + 31) / 32 || g != COLS * ((ng + 31) / 32);   // every tile has a wave
  if (bad) std::printf("E %d groups %d columns %d: %d\n", E, ng, COLS, bad);
  return bad;
}
int main() {
  int bad = 0;
  for (int E = 1; E <= 512; ++E)
    for (int ng = 1; ng <= 64; ++ng) bad += hm::cooc_columns(E) == 2 ? walk<2>(E, ng) : walk<1>(E, ng);
  return bad != 0;
}
""")
    exe = str(tmp_path / "walk")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2508_09591_amd", "csrc"), "-o", exe, str(tmp_path / "walk.cpp")])
    p = subprocess.run([exe], capture_output=True, text=True)
    assert p.returncode == 0, p.stdout[:2000]


def test_selection_asks_for_no_more_lds_than_every_launch_gets(recorder):
    """All hierarchies of the ranks that the call takes, steps that split nothing among them: the counts staged in LDS and the terms of
    64 pairs (four doubles each) beside them stay inside what a kernel has without asking for more, and what fits is staged."""
    result = launch_recorder.run(recorder, r"""
result = []
def chains(G, d, U):
    if len(U) == d:
        yield U
        return
    for u in range(U[-1], G + 1):
        if u % U[-1] == 0 and G % u == 0:
            yield from chains(G, d, U + [u])
for G in (1, 2, 12, 32, 33, 36, 40, 48, 60, 64):
    for d in (1, 2, 3, 4):
        for U in chains(G, d, [1]):
            zi, five = (ctypes.c_void_p * d)(*[at(1).value] * d), (ctypes.c_double * d)(*[0.5] * d)
            rc = L.hm_swap_select(d, (ctypes.c_int32 * d)(*U), G, 64, 8.0, 2.0, zi, at(2), five, 1.0, five, five, 0.1, 0.1, 10.0, at(3), at(4), at(5), at(6),
                                  1 << 30, None)
            result.append([G, U, rc, launched()])
""")
    assert len(result) > 300
    for G, U, rc, launches in result:
        assert rc == 0 and [k["name"] for k in launches] == ["swap_q_kernel<%d>" % (32 if G <= 32 else 64), "swap_argmin_kernel<256>"], (G, U)
        q = launches[0]
        assert q["lds"] + 4 * 64 * 8 <= q["granted"], (G, U, q)
        wanted = [256 * n for n in U[1:] + [G] if n % 4 == 0 and G > 32]
        assert q["lds"] == (sum(wanted) if sum(wanted) + 4 * 64 * 8 <= 65536 else sum(wanted[:3])), (G, U, q)


# A plan of T tokens with a bound of `most` rows per token and, where `rows` is not None, a row count.
_ROWS = r"""
def plan(T, K, most, rows):
    c = B.hm_plan_out()
    c.num_dest, c.row_capacity, c.max_rows_per_token = 32, T * K, most
    c.expected_rows = 0 if rows is None else int(rows * T)
    for i, f in enumerate(("dest_count", "dest_offset", "row_token", "slot_row", "slot_keep", "row_weight", "status")):
        setattr(c, f, at(20 + i).value)
    return ctypes.byref(c)
def kernel(rc):
    assert rc == 0
    one, = launched()
    return one["name"], one["grid"][0]
"""


def test_dispatch_groups_workgroups_by_sizes_alone(recorder):
    """Rows off the line grid: 128 neighbours on one die for rows of 32 bytes or more and up to 80 MB of tokens, 130 MB up to 1,400 bytes a
    row, and at least one whole round of 1,024 workgroups, for each kernel that has the choice and whatever is known of the rows per
    token; whole lines keep the launch order."""
    result = launch_recorder.run(recorder, _ROWS + r"""
result = []
for T, H, off in ((4097, 1030, 0), (38834, 1030, 0), (38835, 1030, 0), (8192, 15, 0), (8192, 17, 0), (92857, 700, 0), (92858, 700, 0), (65000, 701, 0),
                  (65536, 72, 0), (100, 7161, 0), (136, 7161, 0), (137, 7161, 0), (4096, 1024, 16), (4096, 1024, 0), (65536, 100, 0)):
    names = set()
    for most, rows in ((8, None), (0, None), (8, 1.2), (8, 3.0), (8, 5.6), (8, 7.7)):
        x, out = at(1), ctypes.c_void_p(at(2).value + off)
        names.add(kernel(L.hm_dispatch_pack(x, T, 8, H, plan(T, 8, most, rows), out, 8 * T, None)))
    result.append([T, H, off, sorted(names)])   # of kernel and grid
""")
    assert len({n.split("<")[0] for r in result for n, _ in r[3]}) >= 3   # spread_ragged, spread_flat, dispatch_rows
    assert {g >= 1024 for r in result for _, g in r[3]} == {False, True}
    for T, H, off, names in result:
        sizes = (H % 64 != 0 or off != 0) and 2 * H >= 32 and 2 * T * H <= (130e6 if 2 * H <= 1400 else 80e6)
        for name, grid in names:
            assert name.startswith("dispatch_elems") or name.endswith("true>") == (sizes and grid >= 1024), (T, H, off, name, grid)


def test_transpose_reads_eight_rows_for_a_row_count_not_for_a_bound(recorder):
    """Ragged rows: the reads of eight rows in flight for the bf16 transpose of up to eight slots that a row count says are kept nearly all, of
    7 MB or more; four for a plan that was never synchronised, whose bound is eight whatever it holds, and for fp32."""
    result = launch_recorder.run(recorder, _ROWS + r"""
result = []
for T, H in ((16384, 1030), (4097, 1030), (3398, 1030), (3399, 1030), (16384, 2050)):
    for K, most, rows in ((8, 8, None), (8, 0, None), (8, 8, 1.2), (8, 8, 6.9), (8, 8, 7.2), (8, 8, 8), (6, 6, None), (6, 6, 5.8), (5, 5, 4.2), (4, 4, 4), (10, 10, 9.9)):
        for fn, bits in (("hm_combine_transpose_bf16", 16), ("hm_combine_transpose", 32)):
            result.append([T, H, K, rows, bits, kernel(getattr(L, fn)(at(1), T, K, H, plan(T, K, most, rows), at(2), 8 * T, None))[0]])
""")
    for T, H, K, rows, bits, name in result:
        eight = bits == 16 and rows is not None and K <= 8 and rows > max(K - 1, 4.25) and 2 * T * H >= 7e6
        assert name == "spread_ragged_kernel<RowBf16, true, %d, false>" % (8 if eight else 4) if bits == 16 else "RowF32, true, 4" in name, (T, H, K, rows, name)


def test_chunks_of_the_swap_tables_are_summed_by_one_kernel(recorder):
    """Whatever the number of tokens: 16-bit counts of a chunk, up to 16 of them, summed in 32 bits."""
    result = launch_recorder.run(recorder, r"""
result = []
for E in (16, 128, 256):
    for T in (0, 100, 65535, 65536, 522240):
        rc = L.hm_swap_counts(at(1), at(2), T, 8, E, 32, 32, at(3), None, at(4), 1 << 40, None)
        result.append([rc, [k["name"] for k in launched()]])
""")
    for rc, names in result:
        assert rc == 0 and len(names) == 2 and names[1] == "swap_pairs_kernel<unsigned short, 16>", names


def test_counts_take_the_kernel_their_sizes_ask_for(recorder):
    """One kernel of each kind for loads and group counts, and one workgroup only where the owners' table has no room."""
    result = launch_recorder.run(recorder, r"""
result = []
for T, K, E in ((0, 8, 64), (256, 2, 16), (8192, 8, 128), (1024, 64, 4096), (1024, 8, 4097), (600, 8, 8193), (16384, 8, 128), (100001, 1, 256), (30001, 3, 64),
                (70000, 24, 48), (2000000, 1, 4096), (5000, 8, 5000)):
    names = []
    L.hm_expert_load(at(1), at(2), T, K, E, B.hm_topology(4, 8), at(3), at(4), at(5), at(6), None)
    names.append([k["name"] for k in launched()])
    L.hm_group_counts(at(1), at(2), T, K, E, 32, 2, (ctypes.c_int32 * 2)(32, 4), at(3), at(4), None)
    result.append([T, K, E, names + [[k["name"] for k in launched()]]])
""")
    seen = set()
    for T, K, E, both in result:
        for names, what in zip(both, ("load", "group")):
            seen.update(names)
            width = 4 if K >= 4 else 2 if K >= 2 else 1
            alone = T <= 1024 and (E <= 8192 if what == "load" else T * K <= 32768)
            if E > 4096 and alone:
                assert names == ["%s_count_kernel<1024, true>" % what], (T, K, E, names)
            elif E > 4096:
                assert names == ["%s_clear_kernel" % what, "%s_count_kernel<256, false>" % what], (T, K, E, names)
            else:
                assert names in (["%s_owner_kernel<%d, false>" % (what, width)], ["%s_clear_kernel" % what, "%s_owner_kernel<%d, true>" % (what, width)],
                                 ["%s_clear_kernel" % what, "%s_count_kernel<256, false>" % what]), (T, K, E, names)
    assert len(seen) == 2 * (1 + 1 + 1 + 3 + 2), sorted(seen)   # clear, one workgroup, added, spread, whole of two widths


def test_routers_choose_by_lists_wherever_the_lanes_hold_their_experts(recorder):
    """Up to 16 slots, up to 16 groups in a power of two and no softmax with a bias: 8 lanes a token from 16,384 tokens on where they hold the
    experts (512) and the groups, 16 lanes up to 1,024; whatever the number of tokens, no such router takes the kernel of one wave a token."""
    result = launch_recorder.run(recorder, r"""
result = []
for T in (1, 16383, 16384, 65536):
    for E in (1, 64, 512, 513, 768, 1024, 1025, 4096):
        for K in (1, 3, 8, 16, 17):
            for groups in (1, 3, 8, 16, 32):
                for score in (0, 1):
                    for bias in (None, at(4)):
                        if E % groups or K > E:
                            continue
                        r = B.hm_router(E, K, score, groups, groups, 1, 1, 1.0)
                        rc = L.hm_route(at(1), 1, E, bias, T, ctypes.byref(r), at(2), at(3), None)
                        one, = launched()
                        result.append([T, E, K, groups, score, bias is not None, rc, one])
""")
    seen = set()
    for T, E, K, groups, score, biased, rc, one in result:
        lists = K <= 16 and groups in (1, 8, 16) and not (biased and score == 0) and E <= 1024
        lanes = 8 if T >= 16384 and groups <= 8 and E <= 512 else 16
        length = 2 if K <= 2 else 4 if K <= 4 else 8 if K <= 8 else 16
        want = "route_lists_kernel<float, %d, %d>" % (lanes, length) if lists else "route_kernel<float>"
        assert rc == 0 and one["name"] == want, (T, E, K, groups, score, biased, one["name"], want)
        assert one["grid"][0] * (one["block"][0] // (lanes if lists else 64)) >= T and one["lds"] <= one["granted"]
        seen.add(want)
    assert len(seen) == 9


def test_router_calls_of_more_tokens_than_a_launch_has_threads_for(recorder):
    """A launch has less than 2^32 threads: what would need more is refused as a shape, before any launch; the last size that fits is made."""
    result = launch_recorder.run(recorder, _ROWS + r"""
result = []
def note(what, limit, call):
    for T in (limit - 1, limit):
        rc = call(T)
        result.append([what, T == limit, rc, launched()])
def route(T, E, K, groups=1):
    return L.hm_route(at(1), 1, E, None, T, ctypes.byref(B.hm_router(E, K, 0, groups, groups, 1, 1, 1.0)), at(2), at(3), None)
def back(T, E):
    return L.hm_route_backward(at(1), 1, E, at(2), at(3), T, ctypes.byref(B.hm_router(E, 1, 0, 1, 1, 1, 1, 1.0)), at(4), E, None)
note("lists of 8 lanes", (1 << 29) - 31, lambda T: route(T, 8, 1))
note("lists of 16 lanes", (1 << 28) - 15, lambda T: route(T, 600, 2))
note("a wave a token", (1 << 26) - 3, lambda T: route(T, 40, 17))
note("a wave a token, groups", (1 << 26) - 3, lambda T: route(T, 9, 1, 3))
note("gradient of the logits", (1 << 26) - 3, lambda T: back(T, 8))
note("gradient of the logits, rows that fill LDS", (1 << 26) - 3, lambda T: back(T, 4096))
for dtype in (0, 1):
    for H in (8, 5000):
        note("gradient of the weights", (1 << 26) - 3, lambda T: L.hm_combine_weight_grad(at(1), at(2), dtype, T, T, 2, H, plan(T, 2, 2, None), at(5), None))
""")
    assert len(result) == 20
    for what, beyond, rc, launches in result:
        assert (rc, len(launches)) == ((-2, 0) if beyond else (0, 1)), (what, beyond, rc)
        assert all(k["grid"][0] * k["block"][0] < 1 << 32 for k in launches), what


def test_products_up_to_their_limit_are_launched(recorder):
    """(rows / 128 + experts) * ceil(N / 128) up to 2^23 - 8 for every number of rows, also where few rows have more strips of 16 than a
    launch may have workgroups; beyond, HM_ERR_SHAPE without a launch."""
    result = launch_recorder.run(recorder, r"""
result = []
for dtype in (0, 1, 2):
    for E in (1, 2, 32, 100, 1024):
        for rows in (1, 16, 17, 4 * E, 4 * E + 1, 5000, 1 << 20, 1 << 25):
            for N in (1, 4096, 131072, 1 << 20):
                if rows * E < 1 << 35:
                    rc = L.hm_expert_matmul(at(1), at(2), at(3), at(4), at(5), E, rows, N, 256, at(6), dtype, None)
                    result.append([dtype, E, rows, N, rc, launched()])
""")
    seen = set()
    for dtype, E, rows, N, rc, launches in result:
        tiles = (rows // 128 + E) * -(-N // 128)
        if tiles > (1 << 23) - 8:
            assert (rc, launches) == (-2, []) or rc == 0, (dtype, E, rows, N, rc)   # tiles of 256 may fit where those of 128 would not
        else:
            assert rc == 0 and len(launches) == 1, (dtype, E, rows, N, rc)
        for k in launches:
            assert k["grid"][0] <= 1 << 23 and k["grid"][1:] == [1, 1]
            seen.add(k["name"])
    assert any(n.startswith("thin") for n in seen) and len(seen) == 2 + 1 + 3 + 3, sorted(seen)   # few rows; tiles of 256, of 128, of 64


def test_products_take_the_kernel_their_sizes_ask_for(recorder):
    """Strips for up to 32 rows or four an expert; tiles of 64, 128 or, for the unit's 8-bit products, 256; sums as the result's type says."""
    result = launch_recorder.run(recorder, r"""
result = []
for dtype in (0, 1, 2):
    for E, rows, N, side in ((1, 32, 4096, 0), (1, 33, 4096, 64), (8, 32, 2048, 0), (8, 33, 2048, 64), (32, 128, 4096, 0), (32, 129, 4096, 128), (2, 4096, 1000, 128),
                             (4, 2048, 1024, 64), (16, 16384, 1536, 256), (32, 8192, 2048, 128), (32, 65536, 4096, 256)):
        rc = L.hm_expert_matmul(at(1), at(2), at(3), at(4), at(5), E, rows, N, 2048, at(6), dtype, None)
        result.append([dtype, False, side, rc, launched()[0]["name"]])
    for E, N, H, side in ((16, 1536, 2048, 256), (8, 512, 1024, 128), (4, 512, 512, 64)):
        rc = L.hm_expert_matmul_dw(at(1), at(2), at(3), at(4), at(5), E, 4096, N, H, at(6), dtype, None)
        result.append([dtype, True, side, rc, launched()[0]["name"]])
""")
    shape = {64: "2, 1, 1, 2", 128: "2, 2, 2, 2", 256: "4, 4, 2, 2"}
    for dtype, dw, side, rc, name in result:
        out, full = ("float", "true") if dtype == 1 else ("unsigned short", "true" if dtype == 2 else "false")
        if side == 256 and full == "true" and not dw:
            side = 128
        want = "thin_product_kernel<%s>" % out if side == 0 else "product_kernel<%s, %s, %s, %s>" % (shape[side], "true" if dw else "false", full, out)
        assert rc == 0 and name == want, (dtype, dw, side, name, want)


def test_values_in_8_bits_up_to_their_limit_are_launched(recorder):
    """Rows: rows * ceil(C / 512) up to 2^25; columns: (rows / 128 + segments) * ceil(C / 64) up to 2^23; weights of any size."""
    result = launch_recorder.run(recorder, r"""
result = []
for dtype in (0, 1):
    for rows, C, fits in ((1 << 25, 512, 1), ((1 << 25) + 1, 512, 0), (1 << 25, 1, 1), (1 << 24, 513, 1), ((1 << 24) + 1, 513, 0), (1 << 14, 1 << 20, 1)):
        rc = L.hm_quantize_rows(at(1), dtype, C, rows, C, at(2), at(3), None)
        result.append(["rows", fits, rc, launched()])
    for rows, S, C, fits in ((128 * ((1 << 23) - 1), 1, 64, 1), (1 << 30, 1, 64, 0), (127, 512, 1 << 20, 1), (127, 513, 1 << 20, 0)):
        rc = L.hm_quantize_columns(at(1), dtype, C, at(4), S, rows, C, at(2), at(3), None)
        result.append(["columns", fits, rc, launched()])
    for E, N, C in ((1024, 1 << 20, 1 << 20), (1024, 1, 1 << 20), (1, 1 << 20, 1)):
        rc = L.hm_quantize_weights(at(1), dtype, E, N, C, at(2), at(3), at(5), at(6), None)
        result.append(["weights", 1, rc, launched()])
""")
    for what, fits, rc, launches in result:
        assert (rc, len(launches)) == ((0, 1) if fits else (-2, 0)), (what, fits, rc, launches)
        assert all(k["grid"][0] * k["block"][0] < 1 << 32 and max(k["grid"][1:]) < 65536 for k in launches), (what, launches)


def test_swap_tables_take_the_kernels_their_sizes_ask_for(recorder):
    """Matrix products with partial tables, with added ones, and atomics per slot with their tables in LDS and in memory."""
    result = launch_recorder.run(recorder, r"""
result = []
for E, K, G, T, cuts, way in ((128, 8, 32, 8192, [4, 32], "parts"), (256, 9, 32, 8192, [32], "slots"), (256, 8, 32, 522240, [32], "parts"), (256, 8, 32, 522241, [32], "added"),
                              (257, 8, 32, 8192, [32], "added"), (512, 8, 64, 9001, [8, 64], "added"), (513, 8, 32, 8192, [32], "atomics"), (300, 9, 8, 400, [8], "atomics"),
                              (288, 2, 8, 46004, [1, 8], "atomics"), (300, 1, 32, 300000, [4, 32], "atomics"), (64, 1, 8, 523000, [8], "atomics"),
                              (600, 3, 64, 5000, [16, 32, 64], "memory")):
    Z = (ctypes.c_void_p * len(cuts))(*[at(3 + i).value for i in range(len(cuts))])
    rc = L.hm_swap_counts_multi(at(1), at(2), T, K, E, G, len(cuts), (ctypes.c_int32 * len(cuts))(*cuts), Z, at(10), at(11), 1 << 40, None)
    result.append([E, K, T, way, rc, launched()])
""")
    for E, K, T, way, rc, launches in result:
        cols = 2 if 128 < E <= 256 else 1
        want = {"parts": ["swap_cooc_kernel<%d, true, false>" % cols, "swap_pairs_kernel<unsigned short, 16>"],
                "slots": ["swap_slots_kernel", "swap_cooc_kernel<%d, false, false>" % cols, "swap_pairs_kernel<unsigned short, 16>"],
                "added": ["swap_cooc_kernel<%d, true, true>" % cols, "swap_pairs_kernel<int, 1>"]}.get(way, ["swap_factors_kernel", "swap_build_kernel"])
        assert rc == 0 and [k["name"] for k in launches] == ["swap_clear_kernel"] + want, (E, K, T, way, launches)
        assert all(k["lds"] <= k["granted"] for k in launches), launches
        if way in ("atomics", "memory"):
            assert (launches[1]["lds"] > 0) == (way == "atomics"), launches
