"""CPU test of the host code behind the head and shared-prefix calls under AddressSanitizer and
UndefinedBehaviorSanitizer, as ``test_abi_sanitized.py`` does for the others: planning over small,
odd and extreme sizes, and refusals, none of which reaches the GPU."""
import os
import subprocess
import sys
import textwrap

import pytest

from paper_2106_06899_amd import build as b

CHILD = textwrap.dedent(r"""
    import ctypes, itertools, sys
    L = ctypes.CDLL(sys.argv[1])
    i64, vp, i32, f32, sz = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    class Rot(ctypes.Structure):
        _fields_ = [("positions", vp), ("freqs", vp), ("pair_axis", ctypes.c_char_p), ("d_rot", i64), ("axis_stride", i64),
                    ("batch_stride", i64), ("token_stride", i64), ("n_axes", i32), ("position_bytes", i32), ("adjacent", i32), ("inverse", i32)]
    rp = ctypes.POINTER(Rot)
    sigs = {"topk_rope": ([vp, vp] + [i64] * 7 + [rp, i32, vp], i32),
            "topk_qk_norm_rope": ([vp] * 6 + [i64] * 7 + [i32, f32, rp, i32, vp], i32),
            "topk_qk_norm_rope_append": ([vp] * 7 + [i64] * 14 + [i32, f32, rp, i32, vp], i32),
            "topk_qk_norm_rope_backward": ([vp] * 9 + [i64] * 7 + [i32, f32, rp, i32, vp], i32),
            "topk_qk_norm_rope_backward_workspace_bytes": ([i64] * 6 + [i32], sz),
            "topk_attn_prefix": ([vp] * 8 + [i64] * 7 + [vp, i32, f32, i32, vp], i32),
            "topk_attn_prefix_workspace_bytes": ([i64] * 7 + [i32], sz), "topk_last_error": ([], ctypes.c_char_p)}
    for n, (a, r) in sigs.items():
        f = getattr(L, n); f.argtypes = a; f.restype = r
    FAKE, calls, TOP = 0x10000, 0, (1 << 31) - 1
    # planning: every form, from one key and row to the largest
    for B, H, Hkv, Lq in [(1, 1, 1, 1), (4, 12, 12, 1), (3, 15, 3, 1), (64, 32, 8, 1), (16, 16, 4, 5), (40, 12, 12, 1), (8, 8, 1, 10),
                          (1, 24, 3, 33), (4, 16, 4, 512), (2, 2, 2, 129), (1 << 20, 4, 2, 1), (1 << 26, 2, 1, 1), (1, 1 << 27, 1 << 27, 1),
                          (1, 1, 1, 1 << 27)]:
        for P, S in itertools.product([0, 1, 127, 129, 8191, 65536, 1 << 24, TOP], [0, 1, 63, 300, 5000, 1 << 20, TOP]):
            for d in (64, 128):
                n = L.topk_attn_prefix_workspace_bytes(B, H, Hkv, Lq, P, S, d, 1)
                # whole partial results of every row, of 1024 ranges at most
                assert n % (B * H * Lq * (d + 2) * 4) == 0 and n <= 1024 * B * H * Lq * (d + 2) * 4, (B, H, Hkv, Lq, P, S, d, n)
                calls += 1
    for B, T, H, Hkv, d in [(1, 1, 1, 1, 2), (8, 512, 12, 12, 64), (2, 1511, 4, 2, 96), (1, 3, 16384, 16384, 512), (1 << 11, 1 << 20, 1, 1, 64),
                            (1, TOP, 16384, 1, 510), (2, 8192, 32, 8, 128)]:
        for dt, rot in itertools.product((0, 1), (0, 2, d)):
            if rot <= d:
                n = L.topk_qk_norm_rope_backward_workspace_bytes(B, T, H, Hkv, d, rot, dt)
                assert n > 0 and n % (d * 4) == 0, (B, T, H, Hkv, d, rot, n)
                calls += 1
    # refused, each with a message and before anything is launched
    def refused(rc, what):
        global calls
        assert rc < 0 and L.topk_last_error(), what
        calls += 1
    rot = dict(positions=FAKE, freqs=FAKE, pair_axis=None, d_rot=64, axis_stride=0, batch_stride=0, token_stride=1, n_axes=1,
               position_bytes=8, adjacent=0, inverse=0)
    for kw in [dict(d_rot=66), dict(d_rot=3), dict(d_rot=-2), dict(n_axes=0), dict(n_axes=5), dict(positions=None), dict(freqs=FAKE + 4),
               dict(position_bytes=3), dict(adjacent=7), dict(token_stride=-1), dict(batch_stride=1 << 40), dict(n_axes=3, pair_axis=b"\2" * 31 + b"\3")]:
        r = Rot(**dict(rot, **kw))
        refused(L.topk_rope(FAKE, FAKE, 1, 2, 5, 64, 640, 320, 64, r, 1, None), kw)
        refused(L.topk_qk_norm_rope(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1, 5, 2, 1, 64, 1280, 256, 1, 1e-6, r, 1, None), kw)
    for B, T, H, Hkv, d in [(0, 1, 1, 1, 64), (1, 0, 1, 1, 64), (1, 1, 0, 1, 64), (1, 1, 1, 0, 64), (1, 1, 1, 1, 63), (1, 1, 1, 1, 1 << 40),
                            (1 << 62, 1 << 62, 1, 1, 64), (1, 1, 1 << 60, 1, 64), (-5, 1, 1, 1, 64)]:
        refused(L.topk_qk_norm_rope_append(FAKE, None, None, FAKE, FAKE, FAKE, FAKE, B, T, H, Hkv, d, 0, 0, 4, 0, 0, 0, 0, 0, 0, 1, 0.0, None, 1, None), d)
        refused(L.topk_qk_norm_rope_backward(FAKE, None, None, FAKE, FAKE, FAKE, FAKE, None, None, B, T, H, Hkv, d, 0, 0, 1, 0.0, None, 1, None), d)
        assert L.topk_qk_norm_rope_backward_workspace_bytes(B, T, H, Hkv, d, 0, 1) == 0
    for B, H, Hkv, Lq, P, S, d in [(0, 1, 1, 1, 1, 1, 64), (1, 3, 2, 1, 1, 1, 64), (1, 1, 1, 1, -1, 1, 64), (1, 1, 1, 1, 1, 1 << 31, 64),
                                   (1 << 62, 1 << 62, 1, 1, 1, 1, 64), (1, 1, 1, 1 << 62, 1, 1, 64), (1, 1, 1, 1, 1, 1, 96),
                                   (2, 1 << 26, 1 << 26, 1, 0, TOP, 128)]:
        refused(L.topk_attn_prefix(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, B, H, Hkv, Lq, P, S, d, None, 1, 0.125, 1, None), (B, H, P, S))
    print("sanitized head calls:", calls)
""")


def test_host_code_of_heads_and_prefixes_under_sanitizers():
    rt = b.sanitizer_runtime()
    if rt is None:
        pytest.skip("no AddressSanitizer runtime in this ROCm install")
    if not os.path.exists(b.LIB_SAN):
        b.build(variants=("san",))
    env = dict(os.environ, LD_PRELOAD=rt, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-c", CHILD, b.LIB_SAN], env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, f"sanitized run failed ({r.returncode}):\n{r.stdout[-3000:]}\n{r.stderr[-6000:]}"
    assert "sanitized head calls:" in r.stdout
