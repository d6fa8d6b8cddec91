"""CPU test of the host code behind packed attention, the page calls and attention over pages under
AddressSanitizer and UndefinedBehaviorSanitizer, as ``test_abi_sanitized.py`` does for the others:
planning over small, odd and extreme sizes, and refusals, none of which reaches the GPU."""
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
    class Pages(ctypes.Structure):
        _fields_ = [("k", vp), ("v", vp)] + [(n, i64) for n in ("layers", "pages", "heads", "page_rows", "d", "kl", "kp", "kh", "kr", "vl", "vp_", "vh", "vr")]
    pp = ctypes.POINTER(Pages)
    sigs = {"topk_attn_packed": ([vp] * 7 + [i64] * 5 + [vp, i32, f32, i32, vp], i32),
            "topk_attn_packed_backward": ([vp] * 11 + [i64] * 5 + [vp, i32, f32, i32, vp], i32),
            "topk_attn_packed_backward_workspace_bytes": ([i64] * 5 + [i32], sz),
            "topk_attn_tree": ([vp, pp, vp, i64, vp, vp, i64, vp, vp] + [i64] * 4 + [f32, i32, vp], i32),
            "topk_attn_tree_workspace_bytes": ([i64] * 7 + [i32], sz),
            "topk_pages_reserve": ([pp, vp] + [i64] * 3 + [vp] * 3 + [i64, vp, i32, vp], i32),
            "topk_pages_reserve_workspace_bytes": ([i64] * 3, sz),
            "topk_pages_append": ([vp] * 2 + [i64] * 9 + [vp, pp, vp] + [i64] * 3 + [vp, i32, vp], i32),
            "topk_pages_keep": ([pp, vp] + [i64] * 3 + [vp] * 2 + [i64] * 2 + [vp, i32, vp], i32),
            "topk_pages_fork": ([vp] + [i64] * 3 + [vp, i64, vp, vp, i64, vp], i32), "topk_pages_fork_workspace_bytes": ([i64] * 2, sz),
            "topk_pages_release": ([vp] + [i64] * 3 + [vp, i64, vp, i64, vp], i32),
            "topk_pages_compact": ([pp, pp, vp] + [i64] * 3 + [vp] * 4 + [i32, vp], i32), "topk_pages_compact_workspace_bytes": ([i64] * 2, sz),
            "topk_last_error": ([], ctypes.c_char_p)}
    for n, (a, r) in sigs.items():
        f = getattr(L, n); f.argtypes = a; f.restype = r
    FAKE, calls, TOP = 0x10000, 0, (1 << 31) - 1
    HUGE = [0, -1, 1 << 24, 1 << 31, 1 << 40, 1 << 62, (1 << 63) - 1, -(1 << 63)]
    # planning
    for n, N, (H, Hkv), d in itertools.product([1, 3, 64, 65, 1 << 20, 1 << 30], [1, 127, 128, 8193, 1 << 20, 1 << 30], [(1, 1), (12, 12), (16, 4), (80, 16)], (64, 128)):
        x = L.topk_attn_packed_backward_workspace_bytes(n, N, H, Hkv, d, 1)
        assert x == 0 or H * N * 8 <= x <= H * N * 8 + 256 + 8 * 2 * Hkv * N * d * 4, (n, N, H, Hkv, d, x)
        calls += 1
    for B, M, page, (H, Hkv), T, d in itertools.product([1, 7, 300, 1 << 20], [1, 129, 1 << 16, TOP], [1, 16, 100, TOP], [(1, 1), (32, 8), (64, 1)], [1, 13, 64], (64, 128)):
        x = L.topk_attn_tree_workspace_bytes(B, M, page, H, Hkv, T, d, 1)
        assert x <= (1024 + 3 * B) * H * T * (d + 2) * 4 + 8 * B, (B, M, page, H, Hkv, T, d, x)
        calls += 1
    for p, B, M in itertools.product([1, 1000, TOP], [1, 7, 1 << 20], [1, 100, 2000]):
        x = L.topk_pages_reserve_workspace_bytes(p, B, M)
        listed = 0 if p <= 16384 else 4 * p + 4 * -(-p // 4096)  # free pages of large pools
        assert 16 * B + 4 * B * M + listed <= x <= 16 * B + 8 * B * M + 1024 + listed, (p, B, M, x)
        assert L.topk_pages_fork_workspace_bytes(B, M) in (0, 4 * B * (M + 1)) and L.topk_pages_compact_workspace_bytes(p, B) >= 4 * p + 4 * B
        calls += 3
    # refused, each with a message and before anything is launched
    def refused(rc, what):
        global calls
        assert rc < 0 and L.topk_last_error(), what
        calls += 1
    good = dict(k=FAKE, v=FAKE + 64, layers=1, pages=9, heads=2, page_rows=4, d=64, kl=0, kp=512, kh=256, kr=64, vl=0, vp_=512, vh=256, vr=64)
    def every(p, what):
        refused(L.topk_pages_reserve(p, FAKE, 5, 2, 5, FAKE, FAKE, None, 3, FAKE, 1, None), what)
        refused(L.topk_pages_append(FAKE, FAKE, 0, 512, 256, 64, 0, 512, 256, 64, 4, None, p, FAKE, 5, 2, 5, FAKE, 1, None), what)
        refused(L.topk_pages_keep(p, FAKE, 5, 2, 5, FAKE, FAKE, 4, 4, FAKE, 1, None), what)
        refused(L.topk_pages_compact(p, Pages(**dict(good, k=FAKE + 256, v=FAKE + 512)), FAKE, 5, 2, 5, FAKE, FAKE, FAKE, FAKE, 1, None), what)
        refused(L.topk_attn_tree(FAKE, p, FAKE, 5, FAKE, None, 0, FAKE, None, 2, 5, 4, 3, 0.125, 1, None), what)
    for name in ("layers", "pages", "heads", "page_rows", "d"):
        for x in HUGE:
            if (name, x) not in (("pages", 1 << 24), ("page_rows", 1 << 24)):
                every(Pages(**dict(good, **{name: x})), (name, x))
    for name in ("kp", "kh", "kr", "vp_", "vh", "vr"):
        for x in (-1, 7, 1 << 40, (1 << 63) - 8, -(1 << 63)):
            every(Pages(**dict(good, **{name: x})), (name, x))
    for name in ("k", "v"):
        for x in (None, FAKE + 2):
            every(Pages(**dict(good, **{name: x})), (name, x))
    p = Pages(**good)
    for x in [0, -1, 1 << 31, 1 << 62, -(1 << 63), (1 << 63) - 1]:
        refused(L.topk_pages_reserve(p, FAKE, 5, x, 5, FAKE, FAKE, None, 3, FAKE, 1, None), ("B", x))
        refused(L.topk_pages_reserve(p, FAKE, 5, 2, x, FAKE, FAKE, None, 3, FAKE, 1, None), ("M", x))
        refused(L.topk_pages_fork(FAKE, 5, x, 5, FAKE, 9, FAKE, FAKE, 4, None), ("B", x))
        refused(L.topk_pages_fork(FAKE, 5, 2, 5, FAKE, x, FAKE, FAKE, 4, None), ("pages", x))
        refused(L.topk_pages_release(FAKE, 5, 2, x, FAKE, 9, FAKE, 4, None), ("M", x))
        refused(L.topk_pages_release(FAKE, 5, 2, 5, FAKE, 9, FAKE, x, None), ("rows", x))
        refused(L.topk_pages_keep(p, FAKE, 5, 2, 5, FAKE, FAKE, 4, x, FAKE, 1, None), ("A", x))
        refused(L.topk_pages_append(FAKE, FAKE, 0, 512, 256, 64, 0, 512, 256, 64, x, None, p, FAKE, 5, 2, 5, FAKE, 1, None), ("T", x))
        refused(L.topk_attn_tree(FAKE, p, FAKE, 5, FAKE, None, 0, FAKE, None, 2, 5, 4, x, 0.125, 1, None), ("T", x))
        refused(L.topk_attn_tree(FAKE, p, FAKE, 5, FAKE, None, 0, FAKE, None, 2, 5, x, 3, 0.125, 1, None), ("H", x))
        for at in range(4):
            sizes = [2, 100, 4, 2]
            sizes[at] = x
            refused(L.topk_attn_packed(FAKE, FAKE, FAKE, FAKE, FAKE, None, None, *sizes, 64, None, 1, 0.125, 1, None), (at, x))
            refused(L.topk_attn_packed_backward(*[FAKE] * 6, None, *[FAKE] * 4, *sizes, 64, None, 1, 0.125, 1, None), (at, x))
            assert L.topk_attn_packed_backward_workspace_bytes(*sizes, 64, 1) == 0
    print("sanitized page calls:", calls)
""")


def test_host_code_of_packed_and_paged_calls_under_sanitizers():
    rt = b.sanitizer_runtime()
    if rt is None:
        pytest.skip("no AddressSanitizer runtime in this ROCm install")
    if not os.path.exists(b.LIB_SAN):
        b.build(variants=("san",))
    env = dict(os.environ, LD_PRELOAD=rt, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-c", CHILD, b.LIB_SAN], env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, f"sanitized run failed ({r.returncode}):\n{r.stdout[-3000:]}\n{r.stderr[-6000:]}"
    assert "sanitized page calls:" in r.stdout
