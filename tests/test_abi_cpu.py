"""Host-only checks of the C ABI: the library loads, exports every declared
symbol, and its pure-host entry points (schedule, parameter layout, Eq. 1, config
validation) agree with the independent oracle models.  No GPU work is issued."""
import ctypes
import os
import re
from types import SimpleNamespace

import pytest
import torch

from oracle import schedule_oracle as sch
from paper_2503_01328_amd import binding as po
from paper_2503_01328_amd import inputs as syn
from paper_2503_01328_amd import harness

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_declared_symbol_is_exported_and_bound():
    header = open(os.path.join(ROOT, "include", "pipeoffload.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(po_[a-z0-9_]+)\s*\(", header))
    assert len(declared) >= 25
    for name in declared:
        assert hasattr(po.lib, name), f"{name} declared in the header but not exported"
        assert name in po.EXPORTS, f"{name} has no binding"
        assert hasattr(po, name), f"binding lacks a Python function {name}"
    assert set(po.EXPORTS) == declared


SCHEDS = {"1f1b": po.PO_SCHED_1F1B, "1f1b-interleaved": po.PO_SCHED_1F1B_INTERLEAVED}


@pytest.mark.parametrize("name,d,v,m", [("1f1b", 2, 1, 4), ("1f1b", 4, 1, 8), ("1f1b", 8, 1, 16), ("1f1b", 16, 1, 16),
                                        ("1f1b", 4, 1, 3), ("1f1b-interleaved", 8, 2, 32),
                                        ("1f1b-interleaved", 4, 3, 8), ("1f1b-interleaved", 2, 2, 2)])
@pytest.mark.parametrize("ratio", [0.0, 0.25, 0.5, 1.0])
@pytest.mark.parametrize("prefetch", [0, 1, 3])
def test_schedule_ops_match_the_oracle_model(name, d, v, m, ratio, prefetch):
    for rank in sorted({0, d // 2, d - 1}):
        for policy, pname in ((po.PO_SEL_ALTERNATE_MB, "alternate-mb"), (po.PO_SEL_LONGEST_LIFESPAN, "longest-lifespan")):
            got = po.po_schedule_ops(SCHEDS[name], d, rank, v, m, ratio, policy, prefetch)
            passes = sch.compute_passes(name, d, rank, v, m)
            want = sch.with_offload(passes, sch.selected_units(m, v, ratio, pname), prefetch)
            assert got == want
            assert sch.simulate(got)["errors"] == []


@pytest.mark.parametrize("d,v,m,g", [(8, 2, 32, 8), (8, 2, 32, 4), (4, 3, 12, 2), (4, 3, 12, 3), (4, 2, 8, 0), (6, 2, 12, 3),
                                     (2, 1, 4, 1)])
@pytest.mark.parametrize("ratio", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("prefetch", [0, 2, 3])
def test_gis_schedule_ops_match_the_oracle_model(d, v, m, g, ratio, prefetch):
    for rank in sorted({0, d // 2, d - 1}):
        for policy, pname in ((po.PO_SEL_ALTERNATE_MB, "alternate-mb"), (po.PO_SEL_LONGEST_LIFESPAN, "longest-lifespan")):
            got = po.po_schedule_ops(po.PO_SCHED_GIS, d, rank, v, m, ratio, policy, prefetch, group=g)
            passes = sch.compute_passes("gis", d, rank, v, m, g or None)
            want = sch.with_offload(passes, sch.selected_units(m, v, ratio, pname), prefetch)
            assert got == want
            assert sch.simulate(got)["errors"] == []


@pytest.mark.parametrize("name,d,v,m", [("1f1b", 8, 1, 16), ("1f1b-interleaved", 8, 2, 32), ("gis", 8, 2, 32)])
@pytest.mark.parametrize("min_gap", [1, 3, 9])
def test_short_gap_units_are_skipped_like_in_the_oracle_model(name, d, v, m, min_gap):
    code = {"gis": po.PO_SCHED_GIS, **SCHEDS}[name]
    for rank in range(d):
        for ratio in (0.5, 1.0):
            got = po.po_schedule_ops(code, d, rank, v, m, ratio, 0, 2, min_gap=min_gap)
            want = sch.with_offload(sch.compute_passes(name, d, rank, v, m), sch.selected_units(m, v, ratio), 2, min_gap)
            assert got == want


@pytest.mark.parametrize("d,v,m,g", [(8, 2, 32, 0), (8, 2, 11, 4), (8, 4, 16, 6), (4, 3, 7, 2), (4, 4, 16, 4), (6, 3, 18, 0),
                                     (5, 2, 9, 0), (2, 2, 5, 1), (4, 1, 8, 0), (8, 16, 24, 0), (16, 2, 16, 0)])
@pytest.mark.parametrize("ratio", [0.0, 0.5, 1.0])
def test_uniform_repeat_schedule_ops_match_the_oracle_model(d, v, m, g, ratio):
    for rank in sorted({0, d // 2, d - 1}):
        for policy, pname in ((po.PO_SEL_ALTERNATE_MB, "alternate-mb"), (po.PO_SEL_LONGEST_LIFESPAN, "longest-lifespan")):
            for prefetch in (0, 2):
                got = po.po_schedule_ops(po.PO_SCHED_PO, d, rank, v, m, ratio, policy, prefetch, group=g)
                passes = sch.compute_passes("po", d, rank, v, m, g or None)
                want = sch.with_offload(passes, sch.selected_units(m, v, ratio, pname), prefetch)
                assert got == want
                assert sch.simulate(got)["errors"] == []


@pytest.mark.parametrize("d,v,m,g", [(8, 2, 16, 0), (4, 2, 9, 0), (8, 4, 12, 6), (6, 3, 10, 0), (4, 1, 8, 0), (2, 2, 5, 1)])
@pytest.mark.parametrize("k", [0.25, 0.5, 0.9, 1.0, 1.7, 3.0, 40.0])
def test_slot_schedule_ops_match_the_oracle_model(d, v, m, g, k):
    for rank in sorted({0, d // 2, d - 1}):
        for n_sel in range(v + 1):
            got = po.po_schedule_ops_slots(d, rank, v, m, n_sel, k, group=g)
            timed = sch.uniform_repeat_times(d, rank, v, m, g or None)
            placement = sch.slot_placement(timed, set(range(n_sel)), k)
            assert got == sch.with_slot_offload(timed, placement, k)
            assert sch.simulate(got)["errors"] == []


def test_slot_schedule_rejects_bad_arguments():
    for args in [(4, 0, 2, 8, 3, 1.0), (4, 0, 2, 8, 1, 0.0), (4, 0, 2, 8, 1, -1.0), (4, 4, 2, 8, 1, 1.0), (4, 0, 2, 0, 1, 1.0)]:
        with pytest.raises(po.PipeOffloadError) as e:
            po.po_schedule_ops_slots(*args)
        assert e.value.code == po.PO_E_INVAL
    with pytest.raises(po.PipeOffloadError):
        po.po_schedule_ops_slots(8, 0, 2, 8, 1, 1.0, group=3)


def test_uniform_repeat_rejects_bad_groups():
    for g in (3, 9):
        with pytest.raises(po.PipeOffloadError) as e:
            po.po_schedule_ops(po.PO_SCHED_PO, 8, 0, 2, 32, 0.5, group=g)
        assert e.value.code == po.PO_E_INVAL


def test_gis_schedule_rejects_bad_groups():
    for g, m in [(3, 32), (9, 32), (8, 30)]:
        with pytest.raises(po.PipeOffloadError) as e:
            po.po_schedule_ops(po.PO_SCHED_GIS, 8, 0, 2, m, 0.5, group=g)
        assert e.value.code == po.PO_E_INVAL


def test_schedule_ops_reject_bad_arguments():
    for args in [(0, 4, 4, 1, 8, 0.5), (0, 4, 0, 2, 8, 0.5), (1, 4, 0, 2, 6, 0.5), (0, 4, 0, 1, 8, 1.5), (7, 4, 0, 1, 8, 0.5)]:
        with pytest.raises(po.PipeOffloadError) as e:
            po.po_schedule_ops(*args)
        assert e.value.code == po.PO_E_INVAL
        assert "schedule" in po.po_last_error()


def test_grouped_query_layout_and_saved_bytes():
    shape = syn.StageShape(2, 1, 4096, 32, 16384, 4096, dtype="bf16", n_kv_heads=8)
    cfg = harness.make_config(shape)
    layout = {(d["layer"], d["name"]): d for d in po.po_param_layout(cfg)}
    assert (layout[(0, "w_qkv")]["rows"], layout[(0, "w_qkv")]["cols"]) == (4096, 4096 + 2 * 8 * 128)
    assert layout[(1, "b_qkv")]["cols"] == 6144
    assert po.po_param_count(cfg) == 2 * (4096 * 6144 + 6144 + 4096 * 4096 + 2 * 4096 * 16384 + 4096 * 5 + 16384 + 4096)
    model = sch.saved_bytes_per_layer(4096, 4096, 32, 2, 8)
    assert model == (8 * 4096 + 2 * 1024) * 4096 * 2 + 4 * 32 * 4096  # k and v a quarter of the multi-head size
    assert 0 <= po.po_saved_bytes_per_layer(cfg) - model < 6 * 256
    with pytest.raises(po.PipeOffloadError):
        po.po_param_count(harness.make_config(syn.StageShape(2, 1, 4096, 32, 16384, 4096, n_kv_heads=5)))


def test_offload_ratio_for_k():
    assert po.po_offload_ratio_for_k(0.5) == 1.0 and po.po_offload_ratio_for_k(1.0) == 1.0
    assert po.po_offload_ratio_for_k(2.0) == 0.5 and abs(po.po_offload_ratio_for_k(1.6) - 0.625) < 1e-12
    assert po.po_offload_ratio_for_k(0.0) == 1.0 and po.po_offload_ratio_for_k(-1.0) == 1.0


def test_offload_k_is_eq1():
    for h, s in [(8192, 4096), (4096, 4096), (5120, 16384), (2048, 2048)]:
        assert abs(po.po_offload_k(h, s, 220e12, 15e9) - sch.offload_ratio_k(h, s, 220e12, 15e9)) < 1e-12
    assert abs(po.po_offload_k(8192, 4096, 220e12, 15e9) - 0.918) < 1e-3


@pytest.mark.parametrize("key", ["C1", "C2", "C3", "C5"])
def test_param_layout_and_saved_bytes(key):
    shape = syn.CONFIGS[key]
    cfg = harness.make_config(shape)
    layout = po.po_param_layout(cfg)
    h, f = shape.hidden, shape.ffn
    per_layer = 12 * h * h + 13 * h if f == 4 * h else None
    total = po.po_param_count(cfg)
    emb = (shape.vocab + shape.seq) * h if shape.vocab else 0
    assert total == emb + shape.n_layers * per_layer
    # tensors tile the buffer without gaps, in the documented order, 16-byte aligned for bf16
    off = 0
    for d in layout:
        assert d["offset"] == off and d["offset"] % 8 == 0
        off += d["rows"] * d["cols"]
    assert off == total
    names = [d["name"] for d in layout if d["layer"] == 0]
    assert names == [n for n, _ in syn.LAYER_PARAMS]
    # Appendix C: 20 s h bytes per layer at two bytes per element (+ fp32 log-sum-exp, + alignment)
    E = 2 if shape.dtype == "bf16" else 4
    want = sch.saved_bytes_per_layer(shape.seq, h, shape.n_heads, E)
    got = po.po_saved_bytes_per_layer(cfg)
    assert want <= got < want + 6 * 256


def test_invalid_configs_are_rejected_without_touching_the_gpu():
    good = harness.make_config(syn.CONFIGS["C1"])
    assert po.po_param_count(good) > 0
    for field, value in [("n_layers", 0), ("n_chunks", 3), ("hidden", 100), ("n_heads", 7), ("seq", 0),
                         ("dtype", 5), ("rank", 2), ("copy_streams", 3), ("ln_eps", 0.0), ("slot_k", -1.0), ("dropout_p", 1.0),
                         ("group", 5), ("min_gap_passes", -1), ("n_kv_heads", 3), ("weight_stream", 2)]:
        cfg = harness.make_config(syn.CONFIGS["C1"])
        setattr(cfg, field, value)
        with pytest.raises(po.PipeOffloadError) as e:
            po.po_param_count(cfg)
        assert e.value.code == po.PO_E_INVAL


def test_flatten_unflatten_roundtrip():
    shape = syn.StageShape(2, 1, 64, 2, 256, 8, vocab=16, dtype="f32")
    cfg = harness.make_config(shape)
    params = syn.stage_params(shape, 3)
    flat = harness.flatten_params(cfg, params)
    back = harness.unflatten(cfg, flat)
    for l in range(2):
        for k, a in params["layers"][l].items():
            assert (back["layers"][l][k] == a).all()
    assert (back["wte"] == params["wte"]).all() and (back["wpe"] == params["wpe"]).all()


def test_gemm_tile_choice_fills_the_chip():
    """Host logic of the bf16 GEMM: which output tile a shape gets.  The GEMM shapes of the five workloads, the
    grouped-query QKV projection, and shapes that fit no tile."""
    tile = po.po_op_gemm_tile
    # C2 (tokens 2048, h 2048, f 8192): 2048 x 2048 results have only 64 big tiles -> 128 x 128;
    # the QKV projection's 192 big tiles would leave 64 compute units idle -> 256 of the 256 x 192 tiles
    assert tile(2048, 2048) == (128, 128)
    assert tile(2048, 8192) == (256, 256) and tile(8192, 2048) == (256, 256)
    assert tile(2048, 6144) == (256, 192)
    # C3 / C5: whole rounds of big tiles
    assert tile(4096, 4096) == (256, 256) and tile(4096, 12288) == (256, 256) and tile(4096, 16384) == (256, 256)
    assert tile(16384, 15360) == (256, 256) and tile(16384, 5120) == (256, 256) and tile(5120, 15360) == (256, 256)
    # C3 with 8 key/value heads: 384 big tiles need two rounds, 512 narrower ones too, at 3/4 of the work each
    assert tile(4096, 6144) == (256, 192)
    # too few tiles for the big shapes; no 192-wide tile when the row count is no multiple of 256
    assert tile(256, 384) == (128, 128) and tile(128, 6144) == (128, 128) and tile(384, 128) == (128, 128)
    # nothing fits: the shape-generic kernel runs
    assert tile(200, 130) == (0, 0) and tile(64, 64) == (0, 0) and tile(0, 128) == (0, 0)
    for M in range(128, 4097, 128):
        for N in range(64, 6145, 64):
            bm, bn = tile(M, N)
            assert (bm, bn) in ((0, 0), (128, 128), (256, 192), (256, 256))
            assert bm == 0 or (M % bm == 0 and N % bn == 0)


class _Epilogue(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("bias", "residual", "out", "gelu_out", "gelu_u", "acc_f32")] + \
               [("ldc", ctypes.c_int)]


def test_gemm_edge_kernel_leaves_offsets_beyond_31_bits_to_others():
    """Host logic: a lane of the large-tile kernels for any size forms 32-bit byte offsets over a slice of 64 k, also where
    K ends before; the leading dimension of a k-major operand has to leave them room."""
    f = po.lib["_ZN2po24gemm_mfma_edge_supportedEiiiiiPKviS1_iRKNS_8EpilogueE"]
    f.restype = ctypes.c_bool
    f.argtypes = [ctypes.c_int] * 5 + [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_int,
                                       ctypes.POINTER(_Epilogue)]
    at = 1 << 20  # an aligned address; nothing is read
    weight = lambda K, lda, ldb: f(1, 0, 256, 256, K, at, lda, at, ldb, _Epilogue(acc_f32=at, ldc=256))
    forward = lambda K, lda, ldb: f(0, 0, 256, 256, K, at, lda, at, ldb, _Epilogue(out=at, ldc=256))
    most = (1 << 24) - 8  # 64 rows of 2 * most bytes stay below 2^31
    for K in (1, 8, 64):
        assert weight(K, most, 256) and weight(K, 256, most)
        for ld in (1 << 24, 1 << 25, (1 << 25) + 8, 1 << 26, (1 << 30) + 8):
            assert not weight(K, ld, 256) and not weight(K, 256, ld)
    assert forward(64, 64, most) and not forward(64, 64, 1 << 24) and not forward(64, 1 << 23, 256)
    assert weight(4096, 1 << 17, 256) and not weight(4096, 1 << 18, 256)


def test_attention_longer_than_a_grid_goes_to_the_vector_kernels():
    """Host logic: the matrix-core kernels count tiles of rows in the second grid dimension, which ends at 65535."""
    f32, bf16 = (po.lib[n] for n in ("_ZN2po23attention_f32_supportedEPKvS1_iiii", "_ZN2po24attention_mfma_supportedEiiii"))
    f32.restype = bf16.restype = ctypes.c_bool
    f32.argtypes = [ctypes.c_void_p] * 2 + [ctypes.c_int] * 4
    bf16.argtypes = [ctypes.c_int] * 4
    assert f32(1 << 20, 1 << 20, 32 * 65535, 64, 1, 1) and not f32(1 << 20, 1 << 20, 32 * 65535 + 1, 64, 1, 1)
    assert bf16(128 * 65535 - 1, 64, 1, 1) and not bf16(128 * 65535 + 1, 64, 1, 1)
    # fp32: all blocks (32 rows of a head or of a key/value head, 256 threads) in one dimension of 2^32 threads
    assert f32(1 << 20, 1 << 20, 32 * 16, 32 * ((1 << 20) - 2), (1 << 20) - 2, 1)
    assert not f32(1 << 20, 1 << 20, 32 * 16, 32 * ((1 << 20) - 1), (1 << 20) - 1, 1)
    assert f32(1 << 20, 1 << 20, 32 * 65535, 32 * 128, 128, 128) and not f32(1 << 20, 1 << 20, 32 * 65535, 32 * 256, 256, 4)


def test_attention_of_rows_beyond_32_bit_offsets_goes_to_the_vector_kernels():
    """Host logic: the fp32 kernels address 32 rows of 4-byte elements, the ragged bf16 ones 64 rows of 2-byte ones, by 32-bit
    offsets from a tile's first row."""
    f32, bf16 = (po.lib[n] for n in ("_ZN2po23attention_f32_supportedEPKvS1_iiii", "_ZN2po24attention_mfma_supportedEiiii"))
    f32.restype = bf16.restype = ctypes.c_bool
    f32.argtypes = [ctypes.c_void_p] * 2 + [ctypes.c_int] * 4
    bf16.argtypes = [ctypes.c_int] * 4
    at, most = 1 << 20, (1 << 25) - 128  # and two columns of keys and values of 64
    heads = most // 64
    for s in (5, 32, 100):
        assert f32(at, at, s, most, heads, 1) and not f32(at, at, s, most + 64, heads + 1, 1)
        assert not f32(at, at, s, most // 2 + 64, heads // 2 + 1, heads // 2 + 1)
        assert bf16(s, most, heads, 1) and not bf16(s, most + 64, heads + 1, 1)
    assert bf16(128, most + 64, heads + 1, 1)


def test_fp32_gemm_grids_end_below_the_limit_of_a_dimension():
    """Host logic: blocks of 384 and 640 threads pass 2^32 threads at fewer tiles than smaller blocks did; the rest goes to the
    second dimension."""
    class Dim3(ctypes.Structure):
        _fields_ = [(n, ctypes.c_uint32) for n in "xyz"]
    f = po.lib["_ZN2po13gemm_f32_gridEli"]
    f.restype, f.argtypes = Dim3, [ctypes.c_int64, ctypes.c_int]
    for threads in (384, 640):
        for tiles in (1, 256, 3000000, 1 << 24, (1 << 26) + 1, (1 << 31) - 1):
            g = f(tiles, threads)
            assert g.x * threads < 1 << 32 and g.y <= 65535 and g.z == 1
            assert tiles <= g.x * g.y < tiles + g.y
            assert g.y == 1 or tiles * threads > 1 << 31


def test_whole_tiles_of_few_slices_stay_with_the_large_tiles():
    """Host logic: results of whole 128 x 128 tiles take the small ones from K = 256 on where those fill the chip better."""
    f = po.lib["_ZN2po20gemm_small_is_fasterEiii"]
    f.restype, f.argtypes = ctypes.c_bool, [ctypes.c_int] * 3
    for M, N in ((128, 128), (256, 1024), (512, 512), (512, 2048), (1024, 1024), (2048, 512)):
        assert not any(f(M, N, K) for K in (64, 128, 192)) and f(M, N, 256)
    assert f(100, 2048, 64) and f(512, 512, 200)  # no whole tiles, no whole slices


def test_attention_keeps_to_the_faster_of_its_two_kinds_of_blocks():
    """Host logic: calls (rows, head size, heads, key/value heads) which blocks of 32 rows take 3 to 18 percent longer for than those of
    128, and, for every line, one which they take a tenth to a half less for."""
    forward, backward = (po.lib[n] for n in ("_ZN2po31attention_few_forward_is_fasterEiiii",
                                             "_ZN2po32attention_few_backward_is_fasterEiiiii"))
    forward.restype = backward.restype = ctypes.c_bool
    slow = dict(forward=[(410, 64, 40), (421, 64, 37), (1024, 64, 17), (2951, 64, 11), (2550, 128, 11), (2655, 128, 11)],
                backward=[(66, 64, 96), (101, 64, 80), (128, 64, 65), (256, 64, 36), (384, 64, 25), (512, 64, 21), (2048, 64, 9),
                          (2276, 64, 12), (3250, 64, 10), (4090, 64, 8), (74, 128, 96), (99, 128, 80), (896, 128, 13), (1152, 128, 11),
                          (1792, 128, 9), (2304, 128, 7), (2159, 128, 11), (2565, 128, 11), (3572, 128, 8)])
    fast = dict(forward=[(100, 64, 16), (777, 64, 10), (512, 64, 8), (1024, 64, 8), (100, 128, 16), (4096, 128, 2), (777, 128, 10)],
                backward=[(30, 64, 296), (160, 64, 60), (512, 64, 8), (1024, 64, 8), (8190, 64, 3), (100, 128, 16), (2048, 128, 4),
                          (150, 128, 60), (7360, 128, 2)])
    for which, ask in (("forward", forward), ("backward", lambda s, h, a, akv: backward(s, h, a, akv, a // akv))):
        assert not any(ask(s, dh * a, a, a) for s, dh, a in slow[which])
        assert all(ask(s, dh * a, a, a) for s, dh, a in fast[which])
    # groups, whose dK/dV blocks walk several query heads
    assert all(backward(s, dh * a, a, a // hpb, hpb) for s, dh, a, hpb in ((100, 64, 80, 4), (3250, 64, 10, 2), (100, 128, 80, 4)))


@pytest.mark.skipif(torch.cuda.is_available(), reason="forces launches to fail by having no GPU")
@pytest.mark.parametrize("call", ["gemm f32", "gemm bf16", "edge", "attention f32", "attention bf16"])
def test_a_launch_that_cannot_be_set_up_says_so_every_time(call):
    """Without a GPU the LDS size of a kernel cannot be set.  Each such call fails with its own text, and a later one tries
    again instead of remembering the failure."""
    at = 1 << 20  # never read: the call fails on the host
    act = {"gemm f32": lambda: po.po_op_gemm(po.PO_F32, 0, 0, 64, 64, 64, at, 64, at, 64, out=at, stream=0),
           "gemm bf16": lambda: po.po_op_gemm(po.PO_BF16, 0, 0, 256, 256, 256, at, 256, at, 256, out=at, stream=0),
           "edge": lambda: po.po_op_gemm(po.PO_BF16, 0, 0, 1736, 8200, 128, at, 128, at, 8200, out=at, stream=0),
           "attention f32": lambda: po.po_op_attention_forward(po.PO_F32, at, at, at, 64, 64, 1, stream=0),
           "attention bf16": lambda: po.po_op_attention_forward(po.PO_BF16, at, at, at, 100, 64, 1, stream=0)}[call]
    for _ in range(2):
        with pytest.raises(po.PipeOffloadError, match="failed"):
            act()
        with pytest.raises(po.PipeOffloadError, match="unknown dtype"):  # leaves another text behind
            po.po_op_gemm(7, 0, 0, 64, 64, 64, at, 64, at, 64, out=at, stream=0)


def test_hot_kernels_keep_their_accumulators_in_registers():
    """The compiler's own resource report (written by the build): no MFMA kernel may use scratch memory - a GEMM
    whose 256 accumulators spill runs six times slower without failing any numerical test - and the attention
    kernels must still fit two waves per SIMD."""
    import json

    from paper_2503_01328_amd import build as b

    if not os.path.exists(b.RESOURCES):
        b.build(verbose=False)
    usage = json.load(open(b.RESOURCES))
    gemm = {k: v for k, v in usage.items() if "gemm_mfma_kernel" in k}
    grouped = {k: v for k, v in usage.items() if "gemm_mfma_grouped_kernel" in k}
    assert len(grouped) == 1
    attn = {k: v for k, v in usage.items() if "attn_" in k and "_mfma_kernel" in k and "delta" not in k}
    # GEMM: three tiles x four operand layouts x four epilogues; attention: the forward kernel in its two block
    # shapes, the two backward kernels, their eight-wave forms and the one-launch form of both, two head dimensions
    assert len(gemm) == 48 and len(attn) >= 16
    # results of any size: three tiles x (two forward and two input-gradient epilogues, weight gradients) and the grouped
    # launch; the small tiles, bf16 32 x 32 with four waves and 64 x 64 with four, two and one, fp32 32 x 32 with four and eight, x
    # four layouts and the grouped launch, without and with column sums in front; larger fp32 results: three tiles x the same;
    # fp32 16 x 16 tiles: four layouts; fp32 attention: forward, backward and delta, four head sizes; bf16 attention in blocks of
    # 32 rows: forward and backward, two head sizes, sequences of whole 128 rows and others
    edge = {k: v for k, v in usage.items() if "gemm_edge_kernel" in k or "gemm_edge_grouped_kernel" in k}
    small = {k: v for k, v in usage.items() if "gemm_small_kernel" in k or "gemm_small_grouped_kernel" in k}
    gemm_f32 = {k: v for k, v in usage.items() if "gemm_f32_kernel" in k or "gemm_f32_grouped_kernel" in k}
    f32 = {k: v for k, v in usage.items() if "attn_f32_" in k}
    small_sums = {k: v for k, v in usage.items() if "gemm_small_with_sums_kernel" in k}
    f32_sums = {k: v for k, v in usage.items() if "gemm_f32_with_sums_kernel" in k}
    tiny = {k: v for k, v in usage.items() if "gemm_tiny_f32_kernel" in k}
    few = {k: v for k, v in usage.items() if "attn_few_" in k}
    assert len(edge) == 16 and len(small) == 6 * 5 and len(gemm_f32) == 3 * 5 and len(f32) == 12
    assert len(small_sums) == 6 and len(f32_sums) == 3 and len(tiny) == 4 and len(few) == 8
    for name, v in {**gemm, **grouped, **attn, **edge, **small, **small_sums, **gemm_f32, **f32_sums, **tiny, **f32, **few}.items():
        assert v["ScratchSize"] == 0, (name, v)
    for name, v in attn.items():
        assert v["Occupancy"] >= 2, (name, v)
    for name, v in {**gemm, **edge}.items():
        assert v["VGPRs"] + v["AGPRs"] <= 512
    for name, v in {**gemm_f32, **f32_sums}.items():  # two waves of each of three blocks on a SIMD
        assert v["Occupancy"] >= 6, (name, v)
    for name, v in few.items():  # eight waves a block, four in the backward of heads of 128
        assert v["Occupancy"] >= (1 if "attn_few_bwd_kernelILi128" in name else 2), (name, v)
    for name, v in tiny.items():  # eight waves a block
        assert v["Occupancy"] >= 2, (name, v)


def test_trace_viewer_reads_the_span_file(tmp_path):
    """The span file format of PIPEOFFLOAD_TRACE ("# run" separators, "kind start_ms stop_ms" lines) and the viewer."""
    from paper_2503_01328_amd import trace

    f = tmp_path / "t.txt"
    f.write_text("# run\n0 0.0 1.0\n1 1.0 2.5\n# run\n0 0.0 2.0\n0 2.5 3.0\n2 1.0 4.0\n")
    runs = trace.read_runs(str(f))
    assert [len(r) for r in runs] == [2, 3]
    text = trace.render(runs[-1])
    assert "run of 4.00 ms, 3 spans" in text and "compute: 2 spans, busy 2.50 ms" in text
    assert "H2D: 1 spans, busy 3.00 ms" in text and "gap  0.50" in text
    assert trace.main(["trace", str(f), "0"]) == 0 and trace.main(["trace"]) == 2


def test_current_stream_with_and_without_torchs_raw_handle(monkeypatch):
    """The binding asks torch for the current stream's handle by a function that is not public, and does without where there is none."""
    monkeypatch.setattr(po.torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(po, "_raw_stream", lambda device: 100 + device)
    assert po._stream(None) == 103
    monkeypatch.setattr(po, "_raw_stream", None)
    monkeypatch.setattr(po.torch.cuda, "current_stream", lambda: SimpleNamespace(cuda_stream=77))
    assert po._stream(None) == 77
    assert po._stream(5) == 5 and po._stream(SimpleNamespace(cuda_stream=9)) == 9
