"""CPU-only checks of the norm, append and prompt entry points: what the host refuses, and a rotation's fractions of a turn."""
import ctypes
import fractions
import math
import os
import subprocess
import tempfile

import pytest

from test_sanitizers import ENV, ROOT, SAN
from test_serving_host import cache

FAKE = 0x10000000                                            # never dereferenced on the host
LAUNCHED = (0, -5)                                           # (without a GPU a launch fails)


@pytest.fixture(scope="module")
def lib():
    from paper_2502_13652_amd import load_library
    return load_library()


def gpu():
    import torch
    return torch.cuda.is_available()


def test_norm_is_refused(lib):
    from paper_2502_13652_amd.serving import _Norm

    def call(**kw):
        a = dict(x=FAKE, weight=FAKE, out=2 * FAKE, x_stride=64, out_stride=64, rows=4, width=64, dtype=1, weight_dtype=1, residual_dtype=1, out_dtype=1, eps=1e-5)
        a.update(kw)
        return lib.c2t_rms_norm(ctypes.byref(_Norm(**a)), None)
    residual = dict(residual=3 * FAKE, residual_out=4 * FAKE, residual_stride=64, residual_out_stride=64)
    scaled = dict(out_dtype=3, scales=5 * FAKE, scales_stride=2, scale_block=32)
    assert lib.c2t_rms_norm(None, None) == -1
    assert call(rows=0) == 0 and call(rows=0, **residual) == 0 and call(rows=0, **scaled) == 0
    for bad in (dict(rows=-1), dict(width=0), dict(x=None), dict(weight=None), dict(out=None), dict(dtype=3), dict(dtype=7), dict(weight_dtype=2), dict(out_dtype=0), dict(out_dtype=2),
                dict(x_stride=63), dict(out_stride=0), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(residual=FAKE), dict(residual_out=FAKE),
                dict(residual, residual_dtype=2), dict(residual, residual_stride=60), dict(residual, residual_out_stride=-64), dict(out_dtype=3), dict(scales=FAKE), dict(scale_block=32),
                dict(scaled, scale_block=0), dict(scaled, scales_stride=1), dict(scaled, scales=None), dict(out=FAKE, out_stride=128), dict(residual, residual_out=2 * FAKE),
                dict(residual, residual_out=3 * FAKE, residual_out_stride=128), dict(residual, residual_out=FAKE, residual_dtype=0), dict(scaled, out=FAKE)):
        assert call(**bad) == -1, bad
    for big in (dict(width=65537, x_stride=65537, out_stride=65537), dict(x=FAKE + 1), dict(out=2 * FAKE + 1), dict(residual, residual_dtype=0, residual=FAKE + 2), dict(x_stride=1 << 41),
                dict(scaled, scale_block=48), dict(scaled, scale_block=16), dict(scaled, scales=FAKE + 2), dict(scaled, scales_stride=1 << 41), dict(rows=1 << 30)):
        assert call(**big) == -2, big
    if not gpu():
        for fine in (dict(), residual, dict(residual, residual_out=3 * FAKE), dict(residual, residual_out=FAKE), scaled, dict(scaled, scale_block=64), dict(out=FAKE),
                     dict(x=FAKE + 2, x_stride=65, width=63), dict(rows=1 << 24, width=8)):
            assert call(**fine) in LAUNCHED, fine


@pytest.mark.parametrize("kind,bytes_", [("float", 16), ("__bf16", 16), ("_Float16", 16), ("uint8_t", 8)])
def test_pieces_promise_no_more_than_is_asked_for(kind, bytes_, tmp_path):
    """Arrays whose rows begin at multiples of 16 bytes (of 8, of 8 bits) are taken as made of aligned pieces: the pieces' type may not promise the compiler more."""
    source = tmp_path / "piece.hip"
    source.write_text('#include "k_norm.h"\nstatic_assert(alignof(c2t::Eight<%s>) <= %d && sizeof(c2t::Eight<%s>) == 8 * sizeof(%s), "");\n' % (kind, bytes_, kind, kind))
    r = subprocess.run(["hipcc", "-std=c++17", "--offload-arch=gfx950", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2502_13652_amd", "csrc"), str(source)],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout


def test_append_is_refused(lib):
    from paper_2502_13652_amd.serving import _Append

    def call(c=None, **kw):
        a = dict(q=FAKE, k=2 * FAKE, v=3 * FAKE, q_out=4 * FAKE, q_batch_stride=1024, q_token_stride=256, kv_batch_stride=512, kv_token_stride=128, q_out_batch_stride=1024,
                 q_out_token_stride=256, k_out_batch_stride=512, k_out_token_stride=128, turns=FAKE, magnitude=1.0, tokens=4, q_heads=4, layer=0, nodes=0, pairs=32)
        a.update(kw)
        return lib.c2t_cache_append(ctypes.byref(cache(**(c or {}))), ctypes.byref(_Append(**a)), None)
    assert lib.c2t_cache_append(None, ctypes.byref(_Append()), None) == -1 and lib.c2t_cache_append(ctypes.byref(cache()), None, None) == -1
    assert call(c=dict(batch=0)) == -1 and call(c=dict(page_size=7)) == -2 and call(tokens=0) == 0
    tree = dict(nodes=3, position=FAKE)
    for bad in (dict(tokens=-1), dict(q_heads=0), dict(q_heads=3), dict(layer=3), dict(layer=-1), dict(nodes=3), dict(position=FAKE), dict(nodes=5, position=FAKE), dict(nodes=-1),
                dict(q=None), dict(k=None), dict(v=None), dict(q_out=None), dict(turns=None), dict(pairs=0), dict(pairs=4), dict(pairs=40), dict(neighbours=2), dict(magnitude=float("nan")),
                dict(magnitude=float("inf")), dict(tree, starts=FAKE), dict(starts=FAKE, n_new=FAKE), dict(q_token_stride=248), dict(kv_token_stride=120), dict(q_out_token_stride=0),
                dict(k_out=FAKE, k_out_token_stride=64), dict(q_batch_stride=-8), dict(kv_batch_stride=-8), dict(q_out_batch_stride=0), dict(k_out=FAKE, k_out_batch_stride=0),
                dict(q_out=FAKE, q_out_token_stride=512), dict(q_out=FAKE, q_out_batch_stride=2048), dict(k_out=2 * FAKE, k_out_token_stride=256)):
        assert call(**bad) == -1, bad
    for big in (dict(q=FAKE + 8), dict(k=FAKE + 2), dict(v=FAKE + 4), dict(q_out=FAKE + 8), dict(k_out=FAKE + 8), dict(turns=FAKE + 4), dict(q_token_stride=260), dict(kv_batch_stride=516),
                dict(q_out_batch_stride=1028), dict(k_out=FAKE, k_out_token_stride=132), dict(tokens=(1 << 24) + 1), dict(q_batch_stride=1 << 41), dict(tokens=2000, nodes=1025, position=FAKE),
                dict(q_heads=1 << 25, q_token_stride=1 << 31, q_out_token_stride=1 << 31, q_out_batch_stride=1 << 31)):
        assert call(**big) == -2, big
    if not gpu():
        for fine in (dict(), tree, dict(q_out=FAKE), dict(k_out=2 * FAKE), dict(starts=FAKE, q_out_batch_stride=0, q_batch_stride=-3), dict(n_new=FAKE), dict(neighbours=1, pairs=8)):
            assert call(**fine) in LAUNCHED, fine
        assert call(c=dict(batch=1), q_out_batch_stride=0) in LAUNCHED


def test_prompt_is_refused(lib):
    from paper_2502_13652_amd.serving import _Prompt

    def call(**kw):
        a = dict(q=FAKE, k=2 * FAKE, v=3 * FAKE, out=4 * FAKE, q_stride=256, k_stride=128, v_stride=128, out_stride=256, starts=FAKE, rows=100, sequences=2, q_heads=4, kv_heads=2,
                 head_dim=64, dtype=1, scale=0.125)
        a.update(kw)
        return lib.c2t_prompt_attention(ctypes.byref(_Prompt(**a)), None)
    assert lib.c2t_prompt_attention(None, None) == -1 and call(rows=0) == 0
    for bad in (dict(rows=-1), dict(sequences=0), dict(q_heads=0), dict(kv_heads=0), dict(q_heads=3), dict(dtype=3), dict(dtype=-1), dict(q=None), dict(k=None), dict(v=None), dict(out=None),
                dict(starts=None), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q_stride=248), dict(k_stride=120), dict(v_stride=0), dict(out_stride=-256),
                dict(out=FAKE), dict(out=2 * FAKE), dict(out=3 * FAKE)):
        assert call(**bad) == -1, bad
    for big in (dict(dtype=0), dict(head_dim=32), dict(head_dim=96), dict(head_dim=512), dict(sequences=4097), dict(rows=(1 << 24) + 1), dict(q_stride=260), dict(k_stride=(1 << 24) + 8),
                dict(q=FAKE + 8), dict(k=FAKE + 2), dict(v=FAKE + 4), dict(out=4 * FAKE + 8), dict(lse=FAKE + 2), dict(rows=1 << 24, q_heads=4096, kv_heads=4096, q_stride=1 << 18, k_stride=1 << 18,
                v_stride=1 << 18, out_stride=1 << 18)):
        assert call(**big) == -2, big
    if not gpu():
        for fine in (dict(), dict(lse=FAKE), dict(scale=0.0), dict(dtype=2, head_dim=128, q_stride=512, k_stride=256, v_stride=256, out_stride=512), dict(rows=1), dict(rows=1 << 24)):
            assert call(**fine) in LAUNCHED, fine


def test_a_rotations_fractions_of_a_turn():
    """Multiplied by any position they are within 2^-33 of a turn, and its frequencies are the formula's."""
    from paper_2502_13652_amd import Rotation
    pi = fractions.Fraction("3.14159265358979323846264338327950288419716939937510582097")
    f = [10000.0 ** (-2.0 * j / 32) for j in range(16)]
    for r, frequencies in ((Rotation(32, device="cpu"), f), (Rotation(16, frequencies=[0.0, 1.0, -2.5, 1e9, 7.0, 1e-30, 0.1, 3.25], device="cpu"), [0.0, 1.0, -2.5, 1e9, 7.0, 1e-30, 0.1, 3.25])):
        for turn, x in zip(r.turns.tolist(), frequencies):
            for position in (0, 1, -1, 131071, 2 ** 31 - 1, -2 ** 31):
                want = position * fractions.Fraction(x) / (2 * pi)
                got = fractions.Fraction(position * turn % (1 << 64), 1 << 64)
                off = (got - want) % 1
                assert min(off, 1 - off) <= fractions.Fraction(1, 1 << 33)
    for kw in (dict(dim=0), dict(dim=24), dict(dim=-16), dict(dim=16, frequencies=[1.0] * 7), dict(dim=16, frequencies=[math.inf] * 8), dict(dim=16, frequencies=[math.nan] * 8)):
        with pytest.raises(ValueError):
            Rotation(device="cpu", **kw)


def test_layer_entry_points_under_sanitizers():
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, "layer_driver")
        r = subprocess.run(["hipcc", "-O1", "-g", "-std=c++17", "--offload-arch=gfx950",
                            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                            "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                            "-Xarch_host", "-fno-sanitize-recover=all", "-o", exe,
                            os.path.join(SAN, "layer_driver.cpp"), os.path.join(ROOT, "paper_2502_13652_amd", "csrc", "c2t_lib.hip")],
                           stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        assert r.returncode == 0, r.stdout
        r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=ENV)
        assert r.returncode == 0 and "layer driver ok" in r.stdout and "runtime error" not in r.stdout and "AddressSanitizer" not in r.stdout, r.stdout
