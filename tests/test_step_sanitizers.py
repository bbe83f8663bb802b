"""The host code of the calls around the attention, compiled under ASan and UBSan (built as in test_sanitizers.py; no GPU needed)."""
import ctypes
import shutil
import subprocess
from pathlib import Path

import pytest

import paper_2512_23966_amd as loza
from paper_2512_23966_amd import _build
from paper_2512_23966_amd import binding as B

ROOT = Path(__file__).resolve().parent.parent


def test_step_host_code_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    hipcc, clang = shutil.which("hipcc"), shutil.which("amdclang")
    if hipcc is None or clang is None:
        pytest.skip("no hipcc / amdclang")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined"]
    flags = [f for f in _build.HIPCC_FLAGS if f != "-O3"] + ["-O1", "-g"]
    res = subprocess.run([hipcc, *flags, *san, str(_build.CSRC / "ssa_api.hip"), "-o", str(tmp_path / "libloza_ssa_san.so")], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    exe, lib_dir = tmp_path / "sanitize_step", Path(B.LIB_PATH).parent
    subprocess.run([clang, "-std=c99", "-O1", "-g", "-fsanitize=address,undefined", "-I", str(ROOT / "include"), str(ROOT / "tests" / "c" / "sanitize_step.c"),
                    "-o", str(exe), "-L", str(tmp_path), "-lloza_ssa_san", "-L", str(lib_dir), "-lloza_ssa", f"-Wl,-rpath,{tmp_path}", f"-Wl,-rpath,{lib_dir}",
                    "-Wl,-rpath,/opt/rocm/lib"], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr[-3000:]
    got = {line.split()[0]: line.split()[1:] for line in out.stdout.splitlines()}
    big, far = [1, 2, 63, 64, 65, 65536, 2 ** 31 - 1], [1, 64, 8192, 2147483519, 2 ** 63 - 1]
    L, acc = B.lib(), 0
    for b in range(7):
        for h in range(7):
            for n in range(7):
                for x in range(5):
                    pat = (far[(x + b) % 5], far[(x + h) % 5], far[(x + n) % 5])
                    for d in (128, 576):
                        k = ctypes.c_int(0)
                        acc += L.loza_ssa_extend_tree_kernel(big[b], big[h], 1, far[x], big[n], d, *pat, b & 1, ctypes.byref(k)) + k.value
                        acc += L.loza_ssa_extend_tree_workspace_bytes(big[b], big[h], big[h], far[x], big[n], d, 512 if d == 576 else 128, *pat) % 1000
                    acc += L.loza_ssa_verify_tree_workspace_bytes(big[b], big[n], big[h]) % 1000
    assert got["edges"] == [str(acc)]
    freq, m = loza.loza_ssa_rope_frequencies(64, 10000.0, 32.0, 32768)
    assert got["frequencies"][:3] == ["0", "-2", "0"] and float(got["frequencies"][3]) == float(freq[31]) and abs(float(got["frequencies"][4]) - m) < 1e-8
    assert got["refused"] == ["-2"] * 9
