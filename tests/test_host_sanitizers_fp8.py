"""Host layer of the operators of training in 8 bits under AddressSanitizer + UndefinedBehaviorSanitizer:
test_host_sanitizers.py with the program tests/host_sanitize/fp8_driver.cpp, which also walks the plans of the launches (the
runtime's stand-ins turn each of them away)."""
import shutil

import pytest

import test_host_sanitizers as T


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_8_bit_operators_under_asan_and_ubsan(tmp_path, monkeypatch):
    here = tmp_path / "program"
    here.mkdir()
    (here / "driver.cpp").write_text((open(f"{T.HERE}/fp8_driver.cpp").read().replace("../../include", f"{T.ROOT}/include")))
    shutil.copy(f"{T.HERE}/hip_stubs.cpp", here / "hip_stubs.cpp")
    monkeypatch.setattr(T, "HERE", str(here))
    T.test_host_layer_under_asan_and_ubsan(tmp_path)
