"""The host code of norms with rotary positions, token probabilities and pages, compiled under ASan and UBSan (built as in test_step_sanitizers.py; no GPU
needed)."""
import shutil
import subprocess
from pathlib import Path

import pytest

from paper_2512_23966_amd import _build
from paper_2512_23966_amd import binding as B

ROOT = Path(__file__).resolve().parent.parent


def test_host_code_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    hipcc, clang = shutil.which("hipcc"), shutil.which("amdclang")
    if hipcc is None or clang is None:
        pytest.skip("no hipcc / amdclang")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined"]
    flags = [f for f in _build.HIPCC_FLAGS if f != "-O3"] + ["-O1", "-g"]
    res = subprocess.run([hipcc, *flags, *san, str(_build.CSRC / "ssa_api.hip"), "-o", str(tmp_path / "libloza_ssa_san.so")], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    exe, lib_dir = tmp_path / "sanitize_beside", Path(B.LIB_PATH).parent
    subprocess.run([clang, "-std=c99", "-O1", "-g", "-fsanitize=address,undefined", "-I", str(ROOT / "include"), str(ROOT / "tests" / "c" / "sanitize_beside.c"),
                    "-o", str(exe), "-L", str(tmp_path), "-lloza_ssa_san", "-L", str(lib_dir), "-lloza_ssa", f"-Wl,-rpath,{tmp_path}", f"-Wl,-rpath,{lib_dir}",
                    "-Wl,-rpath,/opt/rocm/lib"], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr[-3000:]
    got = {line.split()[0]: line.split()[1:] for line in out.stdout.splitlines()}
    big, far = [1, 2, 63, 64, 65, 1024, 65535, 65536, 2 ** 31 - 1], [1, 2, 64, 8192, 2147483519, 2 ** 31 - 1, 2 ** 63 - 1]
    L, acc = B.lib(), 0
    for a in big:
        for b in big:
            for c in big:
                acc += L.loza_ssa_token_probs_workspace_bytes(a, b, c) % 1000
                acc += sum(L.loza_ssa_norm_rope_backward_workspace_bytes(x, a, b, c) % 1000 for x in far)
    acc += sum(L.loza_ssa_pages_free_workspace_bytes(x) % 1000 + L.loza_ssa_pages_compact_workspace_bytes(x) % 1000 for x in far)
    assert got["edges"] == [str(acc)]
    assert got["refused"] == ["-2"] * 9 and got["overlap"] == ["-2"] * 2
