"""Host logic of the losses behind a first training without a GPU: scratch planning, and refusals that need no context."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

from paper_2601_05732_b200 import binding


def test_scratch_bytes_of_distillation():
    lib = binding.load()
    d, c = lib.mhclite_linear_distill_scratch_bytes, lib.mhclite_linear_ce_scratch_bytes
    for back in (0, 1):
        assert d(64, 100, 1000, 8, back) > c(64, 100, 1000, back) > 0
        assert d(64, 0, 100, 8, back) > 0 and d(64, 100, 1000, 256, back) > 0
        for bad in ((63, 10, 100, 8), (64, -1, 100, 8), (64, 10, 0, 8), (64, 10, 100, 0), (64, 10, 100, 257), (64, 10, 100, -1), (64, 2**30, 2**20, 8)):
            assert d(*bad, back) == 0, bad
    for T in (0, 1, 2**31, 2**62):                        # no size ends the process
        for V in (1, 2**31, 2**62):
            d(64, T, V, 4, 0), d(64, T, V, 4, 1)
    # entries of 16384 x 64: some megabytes on top of the tiles' scratch, whatever the vocabulary
    assert d(2048, 16384, 100000, 64, 1) - c(2048, 16384, 100000, 1) < 32 << 20


def test_scratch_bytes_of_sequences():
    lib = binding.load()
    p, q = lib.mhclite_policy_scratch_bytes, lib.mhclite_preference_scratch_bytes
    assert p(1, 1) == p(0, 3) == q(1000, 4) == 0                 # a handful of tokens needs none
    assert p(10, 1000) > 0 and q(100000, 4) == p(100000, 8) > 0
    for bad in ((-1, 3), (10, -1), (2**31, 3), (2**62, 3), (10, 2**30), (10, 2**62)):
        assert p(*bad) == 0 and q(*bad) == 0, bad
    assert q(100000, 2**29) == 0 and p(2**31 - 257, 2**30 - 1) > 0
    # a byte for four tokens, 28 a sequence; the pieces' number has a bound
    assert p(2**24, 1000) < (2**24 // 4) + 64 * 1000 + (1 << 20)


def test_null_context_is_refused():
    lib = binding.load()
    names = [n for n in binding.SIGNATURES if n.startswith(("mhclite_linear_distill", "mhclite_policy", "mhclite_preference")) and not n.endswith("_bytes")]
    assert len(names) == 4
    for name in names:
        zero = [0.0 if a in (ctypes.c_float, ctypes.c_double) else None if a is ctypes.c_void_p else 0 for a in binding.SIGNATURES[name][1]]
        assert getattr(lib, name)(*zero) == binding.ERR_BAD_ARG, name


def test_arguments_are_refused_before_the_library_sees_them():
    m = binding.load_marshal()
    c = m.make(1234, 0, 4, 64)                            # a handle that no call gets as far as using
    bf, f32, i64 = (lambda *s, t=t: torch.zeros(*s, dtype=t) for t in (torch.bfloat16, torch.float32, torch.int64))
    out = (f32(3), f32(3), f32(3, 5))
    value = [(m.linear_distill_fwd, bf(3, 64), bf(9, 64), i64(3), f32(3, 5), 1.0, 1.0, *out),             # one axis
             (m.linear_distill_fwd, bf(3, 64), bf(9, 63), i64(3, 5), f32(3, 5), 1.0, 1.0, *out),
             (m.linear_distill_fwd, bf(3, 64), bf(9, 64), i64(3, 5), f32(3, 5), 1.0, 1.0, *out),           # not on the device
             (m.policy_loss, f32(9), f32(9), None, i64(9), i64(3), f32(2), False, 0.2, 0.2, 0.0, True, f32(2), f32(2, 3), None, None),
             (m.preference_loss, f32(9), None, i64(9), i64(3), 0.1, 0.0, 0.0, True, f32(1), f32(1, 2), None, None)]
    kind = [(m.linear_distill_fwd, None, bf(9, 64), i64(3, 5), f32(3, 5), 1.0, 1.0, *out), (m.linear_distill_bwd, bf(3, 64)),
            (m.policy_loss, f32(9)), (m.preference_loss, 3, None, i64(9), i64(3), 0.1, 0.0, 0.0, True, f32(1), f32(1, 2), None, None),
            (m.linear_distill_fwd, bf(3, 64), 7, i64(3, 5), f32(3, 5), 1.0, 1.0, *out)]
    for error, calls in ((ValueError, value), (TypeError, kind)):
        for f, *args in calls:
            with pytest.raises(error):
                f(c, *args)
    with pytest.raises(ValueError, match="closed"):
        m.linear_distill_fwd(None, bf(3, 64), bf(9, 64), i64(3, 5), f32(3, 5), 1.0, 1.0, *out)


def test_included_kernels_do_not_read_by_the_read_only_path():
    """Kernels that begin while their predecessor runs, kept in files that others include (csrc/kernels.h tells why)."""
    csrc = os.path.join(os.path.dirname(binding.__file__), "csrc")
    seen = 0
    for name in sorted(os.listdir(csrc)):
        src = re.sub(r"//[^\n]*", "", open(os.path.join(csrc, name)).read())
        if "launch_after(" in src and name.endswith(".cuh"):
            seen += 1
            assert src.count("pdl_wait();") == src.count("__global__"), name
            for word in ("__ldg", "__ldcg", ".nc.", "ld_stream(", "__restrict__"):
                assert word not in src.replace("ld_dep_stream(", ""), (name, word)
    assert seen >= 1


def test_token_indices_up_to_the_largest_count(tmp_path):
    """T may be 2^31 - 257, so a walk looks for tokens whose index no 32-bit number holds.  In a constant expression a signed
    overflow is an error of the compiler's: the questions asked of indices are asked here for the steps next to the end, with the
    answers of Python's unbounded integers."""
    csrc = os.path.join(os.path.dirname(binding.__file__), "csrc")
    lines = []
    for T in (1, 127, 128, 129, 2**31 - 641, 2**31 - 512, 2**31 - 511, 2**31 - 384, 2**31 - 383, 2**31 - 257):
        for base in range((T - 1) // 128 * 128, -1, -128)[:6]:
            for n in (0, 128, 256, 384, 512):
                yes = ("!", "")
                lines.append(f"static_assert({yes[base + n < T]}mhcl::seq_before({base}, {n}, {T}), \"\");")
                lines.append(f"static_assert({yes[base + n <= T]}mhcl::seq_whole({base}, {n}, {T}), \"\");")
    src = tmp_path / "index.cpp"
    src.write_text('#include "seq_index.h"\n' + "\n".join(lines) + "\n")
    r = subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-fsyntax-only", f"-I{csrc}", str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[:2000]
    # and the kernels ask them so: no sum of an index and steps is compared with the end
    kernels = re.sub(r"//[^\n]*", "", open(os.path.join(csrc, "seq_losses.cuh")).read())
    assert not re.findall(r"\+ [\w *()-]*k(?:SeqStep|ScaleRange)\)* *[<>]=? *(?:a\.T|hi)\b", kernels)
    assert kernels.count("seq_before(") >= 4 and kernels.count("seq_whole(") >= 4
