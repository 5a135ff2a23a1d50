"""The 8-bit key/value cache and the rotary positions without a GPU: rules that host and device share (csrc/kv8.h) and refusals of the entry
points under the sanitizers, the plan of the rotary positions against its formulas, and what the binding refuses."""
import ctypes
import math
import os
import shutil
import subprocess

import pytest
import torch

from paper_2604_06832_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2604_06832_amd")
BUILD = os.path.join(PKG, "_build")
HIPCC = "/opt/rocm/bin/hipcc"
CLANG = "/opt/rocm/lib/llvm/bin/clang++"
OTHER_UNITS = ["bd_lib", "k_stream", "k_mega", "k_prefill", "k_attention"]


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__ as g
        g.build()


def _run(cmd):
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, " ".join(cmd) + "\n" + r.stdout[-4000:]
    return r.stdout


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)), reason="no ROCm compiler here")
def test_shared_rules_and_refusals_under_asan_and_ubsan(tmp_path):
    if not all(os.path.exists(os.path.join(BUILD, u + ".o")) for u in OTHER_UNITS):
        import __graft_entry__ as g
        g.build()
    d = str(tmp_path)
    _run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Wno-unused-value", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
          "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined",
          "-c", os.path.join(PKG, "csrc", "k_kv8.hip"), "-o", os.path.join(d, "k_kv8.o")])
    _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-shared-libsan",
          os.path.join(d, "k_kv8.o"), *[os.path.join(BUILD, u + ".o") for u in OTHER_UNITS], "-o", os.path.join(d, "libbd_san.so")])
    rt = os.path.dirname(_run([CLANG, "-print-file-name=libclang_rt.asan-x86_64.so"]).strip())
    _run([HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-g", "-O1", "-Wno-unused-value", "-Xarch_host", "-fsanitize=address", "-Xarch_host",
          "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined", "-shared-libsan", os.path.join(ROOT, "tests", "kv8_rules_check.cpp"),
          "-L" + d, "-lbd_san", "-Wl,-rpath," + d, "-Wl,-rpath," + rt, "-o", os.path.join(d, "check")])
    # (what the ROCm runtime keeps until the process ends is not the library's)
    r = subprocess.run([os.path.join(d, "check")], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300,
                       env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1"))
    shutil.rmtree(d, ignore_errors=True)
    assert r.returncode == 0 and "ALL OK" in r.stdout, r.stdout[-3000:]
    assert "ERROR: AddressSanitizer" not in r.stdout and "runtime error:" not in r.stdout, r.stdout[-3000:]


@pytest.mark.parametrize("scaling", [binding.BD_ROPE_PLAIN, binding.BD_ROPE_LINEAR, binding.BD_ROPE_BASE, binding.BD_ROPE_PARTS])
@pytest.mark.parametrize("D,R,theta,factor,trained", [(128, 128, 1e6, 4.0, 8192), (64, 34, 1e4, 8.5, 2048), (128, 4, 5e5, 1.0, 1), (64, 64, 1e6, 32.0, 1 << 20)])
def test_plan_of_rotary_positions(scaling, D, R, theta, factor, trained):
    plan = binding.bd_k_rope_plan(D, R, binding.BD_ROPE_INTERLEAVED, theta, scaling, factor, trained)
    assert (plan.D, plan.rotary_dim, plan.layout) == (D, R, binding.BD_ROPE_INTERLEAVED)
    for i in range(R // 2):
        f = math.exp(-2.0 * i / R * math.log(theta))
        if scaling == binding.BD_ROPE_LINEAR:
            f /= factor
        elif scaling == binding.BD_ROPE_BASE:
            f *= math.exp(-2.0 * i / (R - 2) * math.log(factor))          # (theta s^(R/(R-2)))^(-2i/R)
        elif scaling == binding.BD_ROPE_PARTS:
            w = min(max((trained * f / (2 * math.pi) - 1) / 31, 0.0), 1.0)
            f = w * f + (1 - w) * f / factor
        assert abs(plan.inv_freq[i] - f) <= 1e-14 * f * max(1.0, math.log(theta))
    assert abs(plan.amplitude - (1 + 0.1 * math.log(factor) if scaling == binding.BD_ROPE_PARTS else 1)) <= 2.0 ** -23
    if scaling == binding.BD_ROPE_BASE:                                    # the slowest pair is stretched by the factor, the fastest not at all
        plain = binding.bd_k_rope_plan(D, R, 0, theta)
        assert plan.inv_freq[0] == 1.0 and abs(plain.inv_freq[R // 2 - 1] / plan.inv_freq[R // 2 - 1] / factor - 1) < 1e-12


def test_plan_refusals_reach_python():
    for args in ((96, 64), (64, 65), (64, 128)):
        with pytest.raises(binding.BdError) as e:
            binding.bd_k_rope_plan(*args)
        assert e.value.code == binding.BD_E_ARG


def test_binding_takes_no_host_tensors():
    pages, lens = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        binding.Kv8Cache(torch.zeros((2, 1, 4096), dtype=torch.uint8), torch.zeros((2, 1), dtype=torch.int32), pages, lens)
    with pytest.raises(ValueError):
        binding.bd_k_rope(binding.bd_k_rope_plan(64), torch.zeros((1, 1, 1, 64)), lens)


def test_a_cache_keeps_the_tensors_that_its_pointers_belong_to():
    """Changing a tensor in place is fine; another tensor in its place is refused, since the kernels would go on with the old one's memory."""
    c = binding.Kv8Cache.__new__(binding.Kv8Cache)
    for name in ("codes", "scales", "pages", "lens", "status"):
        t = torch.zeros(3, dtype=torch.int32)
        setattr(c, name, t)
        with pytest.raises(AttributeError):
            setattr(c, name, t + 1)
        with pytest.raises(AttributeError):
            setattr(c, name, None)
        assert getattr(c, name) is t
    c.lens += 4
    assert c.lens.tolist() == [4, 4, 4]
    c.n_seq = 3
    with pytest.raises(AttributeError):
        c.n_seq = 2


BIG = 1 << 32


@pytest.mark.parametrize("change", [{"n_q": BIG + 4}, {"M": BIG + 4}, {"window": BIG + 8}, {"window": 8 - BIG}, {"sinks": BIG + 4}, {"sinks": 4 - BIG}])
def test_workspace_refuses_numbers_past_32_bits(change):
    """(ctypes would cut them to 32 bits and ask for another call's workspace.)"""
    one = torch.zeros(64, dtype=torch.int32)
    c = binding.Kv8Cache.__new__(binding.Kv8Cache)
    c._c = binding.bd_kv8(one.data_ptr(), one.data_ptr(), one.data_ptr(), one.data_ptr(), None, 4, 2, 64, 2, 4096)
    c._p, c._workspace = ctypes.addressof(c._c), binding.lib().bd_k_kv8_attention_workspace
    call = {"n_q": 4, "M": 4, "window": 0, "sinks": 0}
    assert c.bd_k_kv8_attention_workspace(**call) > 0
    with pytest.raises(ValueError):
        c.bd_k_kv8_attention_workspace(**{**call, **change})


@pytest.mark.parametrize("change", [{"D": BIG + 64}, {"rotary_dim": BIG + 32}, {"layout": BIG}, {"layout": 1 - BIG}, {"scaling": BIG + 1}, {"trained": BIG + 4096}])
def test_plan_refuses_numbers_past_32_bits(change):
    call = {"D": 64, "rotary_dim": 32, "layout": 0, "scaling": binding.BD_ROPE_PARTS, "factor": 2.0, "trained": 4096}
    binding.bd_k_rope_plan(**call)
    with pytest.raises(ValueError):
        binding.bd_k_rope_plan(**{**call, **change})


def test_a_short_workspace_says_so_without_a_gpu(monkeypatch):
    """(a refused call looks at no memory)"""
    mem = torch.zeros(64, dtype=torch.int32)
    p = mem.data_ptr() + -mem.data_ptr() % 16
    c = binding.bd_kv8(p, p, p, p, None, 4, 2, 64, 2, 4096)
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    monkeypatch.setattr(binding, "_current_stream", lambda index: None)
    with pytest.raises(binding.BdError, match="bytes of workspace, got 16") as e:
        binding._enqueue(0, binding.lib().bd_k_kv8_attention, (ctypes.addressof(c), p, 1024, 256, 4, 4, None, binding.BD_MODE_CAUSAL, 0, 0, 0.0, p, 1024, 256, p, 16))
    assert e.value.code == binding.BD_E_CAPACITY and "capacity exceeded" not in str(e.value)
