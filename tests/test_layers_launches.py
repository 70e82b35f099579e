"""The layer operators' launches at the largest sizes whose matrices the card's 288 GB hold: a launch takes fewer than 2^32 threads.  Host code
only, against a stand-in for the HIP runtime; the pointers are never followed."""
import os
import subprocess
import sys
import textwrap

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(os.path.dirname(HERE), "paper_2502_17846_amd", "libgrem.so")

BODY = """
import ctypes, sys
fake = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
sys.path.insert(0, sys.argv[2])
ctypes.CDLL(sys.argv[3])                          # (its kernels first: torch has more than the stand-in keeps names of)
from paper_2502_17846_amd import binding as B
fake.fake_text.restype = ctypes.c_char_p
lib = B.load()
P, ROOM = 1 << 20, 288 * 10 ** 9
ws = ctypes.c_size_t(1 << 62)
seen = set()

def sizes(tall):
    return [1 << 30, (1 << 30) - 1, 1 << 29, 1 << 27, 10 ** 6 + 1, 300, 1] if tall else [1 << 20, (1 << 20) - 1, 65_537, 16_384, 4_097, 256, 100, 1]

def check(what):
    for line in fake.fake_text().decode().splitlines():
        kind, name, threads = line.rsplit(" ", 1)[0].split(" ", 1) + [int(line.rsplit(" ", 1)[1])]
        if kind == "launch":
            seen.add(name)
            assert 0 < threads < 1 << 32, (what, name, threads)
    fake.fake_reset(ctypes.c_size_t(1 << 62))

def rows(d, ck=False):
    return ctypes.byref(B.Rows(P, d, P if ck else None, -(-d // 32) if ck else 0))

fake.fake_reset(ctypes.c_size_t(1 << 62))
for t, size in ((0, 4), (1, 2), (2, 2)):
    for n in sizes(True):
        for d in sizes(False):
            if 2 * n * d * size > ROOM:
                continue
            for labels in (None, P):
                for nnz in (0, 10 ** 10):
                    assert lib.grem_neighbour_mean(P, 64, P, nnz, n, labels, t, d, P, d, P, d, P, P, ws, None) == 0
                    assert lib.grem_neighbour_mean_backward(P, 64, P, nnz, n, labels, P, t, d, P, d, P, d, P, ws, None) == 0
                    check(("mean", t, n, d, nnz))
            assert lib.grem_layer_norm(t, n, d, P, d, P, P, 1e-5, P, d, P, P, None) == 0
            assert lib.grem_layer_norm_backward(t, n, d, P, d, rows(d), P, P, P, P, d, P, P, P, ws, None) == 0
            assert lib.grem_checkpoint_pack(t, n, d, P, d, P, d, P, -(-d // 32), None) == 0
            assert lib.grem_checkpoint_unpack(t, n, d, rows(d, True), P, d, None) == 0
            check(("rows", t, n, d))
            for m in sizes(False):
                for kb in (0, d):
                    if (n * (d + kb) + n * m + m * (d + kb)) * size > ROOM:
                        continue
                    width = d + kb
                    assert lib.grem_linear(t, n, m, P, d, d, P, kb, kb, P, width, P, 1, None, 0, P, m, None, 0, None) == 0
                    check(("linear", t, n, d, kb, m))
                    for act in (0, 3):
                        if lib.grem_linear_backward_bytes(t, n, m, d, kb, act) > ROOM:
                            continue
                        assert lib.grem_linear_backward(t, n, m, P, m, act, P, m, rows(d), d, rows(kb), kb, P, width, P, d, P if kb else None, kb, P, width,
                                                        P, P, ws, None) == 0
                        check(("linear backward", t, n, d, kb, m))
for part in ("k_nm_rows", "k_nm_segments", "k_nm_order", "k_lin_direct", "k_lin_weight", "k_lin_prepare", "k_lin_join", "k_ln_forward", "k_ln_columns_wide",
             "k_ck_pack"):
    assert any(part in name for name in seen), part
print("launches:", len(seen))
"""


def test_threads(tmp_path):
    out = str(tmp_path / "libamdhip64.so.7")
    subprocess.run(["gcc", "-shared", "-fPIC", "-O1", "-w", "-Wl,-soname,libamdhip64.so.7", "-o", out, os.path.join(HERE, "fake_grids.c")], check=True)
    if not os.path.exists(LIB):
        from paper_2502_17846_amd import build
        build.build_library()
    done = subprocess.run([sys.executable, "-c", textwrap.dedent(BODY), out, os.path.dirname(HERE), LIB], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stdout + done.stderr[-3000:]
