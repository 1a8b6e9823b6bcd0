"""Host logic of the operators around the stack without a GPU: scratch planning and refusals that need no context."""
import ctypes
import os
import re
import subprocess
import sys

import pytest
import torch

from paper_2601_05732_b200 import binding


def test_scratch_bytes():
    lib = binding.load()
    e, b, c = lib.mhclite_embed_scratch_bytes, lib.mhclite_block_scratch_bytes, lib.mhclite_linear_ce_scratch_bytes
    assert e(64, 10, 100) == 0 and e(64, 100000, 100) > e(64, 1000, 100) > 0      # a handful of tokens needs none
    assert e(63, 10, 100) == 0 and e(64, -1, 100) == 0 and e(64, 10, 0) == 0
    assert b(64, 0) == 0 and b(4096, 100000) > b(4096, 8) > 0 == b(4096, 1) and b(16392, 8) == 0 and b(65, 8) == 0
    assert c(64, 10, 100, 0) > 0 and c(64, 10, 0, 0) == 0 and c(12, 10, 100, 1) == 0
    for T in (0, 1, 2**31, 2**62):                        # no size ends the process
        for V in (1, 2**31, 2**62):
            e(64, T, V), b(64, T), c(64, T, V, 0), c(64, T, V, 1)
    assert c(64, 2**30, 2**20, 1) == 0 and c(64, 0, 100, 1) > 0
    # the logits of 16384 tokens over 100 000 words would be 3.3 GB in bf16; the backward holds a piece of them
    assert c(2048, 16384, 100000, 1) < 600 << 20
    assert c(2048, 16384, 100000, 0) < 200 << 20


def test_null_context_is_refused():
    lib = binding.load()
    for name, (_, args) in binding.SIGNATURES.items():
        if name.startswith(("mhclite_embed", "mhclite_block", "mhclite_dropout", "mhclite_linear_ce", "mhclite_set_status")):
            if name.endswith("_bytes"):
                continue
            zero = [0.0 if a is ctypes.c_float else None if a is ctypes.c_void_p else 0 for a in args]
            assert getattr(lib, name)(*zero) == binding.ERR_BAD_ARG, name
    assert binding.status_string(binding.ERR_INDEX) not in ("ok", "unknown status")


def test_arguments_are_refused_before_the_library_sees_them():
    m = binding.load_marshal()
    c = m.make(1234, 0, 4, 64)                            # a handle that no call gets as far as using
    bf, f32, i64 = (lambda *s, t=t: torch.zeros(*s, dtype=t) for t in (torch.bfloat16, torch.float32, torch.int64))
    value = [(m.dropout, f32(3), 0.1, None, None), (m.dropout, bf(3), 0.1, None, None),            # type, then device
             (m.block_in_fwd, bf(3, 65), f32(64), 1e-6, bf(3, 64), f32(3)), (m.block_in_fwd, bf(()), f32(64), 1e-6, bf(64), f32(1)),
             (m.embed_fwd, i64(3, 1), bf(9, 64), 1.0, bf(3, 4, 64)), (m.embed_bwd, i64(3), bf(3, 4, 64), 1.0, f32(()), False),
             (m.linear_ce_fwd, bf(3, 64), bf(9, 63), i64(3), 1.0, f32(3), f32(3))]
    kind = [(m.dropout, 3, 0.1, None, None), (m.dropout, bf(3)), (m.linear_ce_bwd, bf(3, 64), None, None, 1.0, None, None, None, None)]
    for error, calls in ((ValueError, value), (TypeError, kind)):
        for f, *args in calls:
            with pytest.raises(error):
                f(c, *args)
    with pytest.raises(ValueError, match="closed"):
        m.dropout(None, bf(3), 0.1, None, None)
    with pytest.raises(ValueError):
        m.dropout(object(), bf(3), 0.1, None, None)
    with pytest.raises(KeyError):
        m.bind({})


def test_status_words_are_never_shared_or_given_back(monkeypatch):
    class Torch:                                          # device memory of the host
        int32 = torch.int32
        empty = staticmethod(lambda *s, dtype, device: torch.empty(*s, dtype=dtype))
    monkeypatch.setattr(binding, "_status_slabs", {})
    rows = [binding._status_words(Torch, d).data_ptr() for _ in range(300) for d in (0, 1)]      # the tensors are dropped
    assert len(set(rows)) == 600 and all(r % 16 == 0 for r in rows)
    held = {s.data_ptr() + 32 * i for slabs, _ in binding._status_slabs.values() for s in slabs for i in range(len(s))}
    assert set(rows) <= held


def test_overlapped_kernels_do_not_read_by_the_read_only_path():
    """A kernel launched while its predecessor runs must not promise that nobody writes what it reads (csrc/kernels.h)."""
    csrc = os.path.join(os.path.dirname(binding.__file__), "csrc")
    launched = 0
    for name in sorted(os.listdir(csrc)):
        src = re.sub(r"//[^\n]*", "", open(os.path.join(csrc, name)).read())
        if name == "philox.cuh" or "launch_after(" in src and name.endswith(".cu"):
            launched += 1
            for word in ("__ldg", "__ldcg", ".nc.", "ld_stream(", "__restrict__"):
                assert word not in src.replace("ld_dep_stream(", ""), (name, word)
    assert launched == 4


def test_contexts_do_without_the_extension_until_a_call_needs_it(monkeypatch):
    class Lib:
        def __getattr__(self, name):
            return lambda *a: 0

    def missing():
        raise ImportError("no extension here")
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(binding, "load", Lib)
    monkeypatch.setattr(binding, "_status_words", lambda t, d: torch.zeros(8, dtype=torch.int32))
    monkeypatch.setattr(binding, "load_marshal", missing)
    c = binding.MhcLite(4, 64)
    c.set_kernel_timing(True)
    with pytest.raises(ImportError, match="no extension here"):
        c.dropout(torch.zeros(3), 0.1, None, None)
    with pytest.raises(AttributeError):
        c.no_such_call

    class Module:
        make = staticmethod(lambda *a: a)
        dropout = staticmethod(lambda c, *a: seen.append(c) or 0)
    seen = []
    monkeypatch.setattr(binding, "load_marshal", lambda: Module)
    c._h.value = 77
    c.dropout(None, 0.1, None, None)
    c.close()
    c.dropout(None, 0.1, None, None)
    assert seen == [(77, 0, 4, 64), None]                 # a closed context is passed as such
    d = binding.MhcLite(4, 64)
    d._h.value = 78
    d.close()                                             # closed before its first call
    d.dropout(None, 0.1, None, None)
    assert seen[2] is None


def test_extension_built_against_another_torch_is_built_anew():
    code = """
import torch
torch.__version__ = "0.0"
from paper_2601_05732_b200 import binding, build
calls = []
build.build_marshal = lambda force=False: calls.append(force)
try:
    binding.load_marshal()
except ImportError as e:
    assert "built against torch" in str(e) and len(calls) == 1
else:
    raise SystemExit("an extension of another torch was loaded")
"""
    root = os.path.dirname(os.path.dirname(binding.__file__))
    subprocess.run([sys.executable, "-c", code], cwd=root, check=True, timeout=300)
