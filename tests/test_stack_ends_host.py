"""Host logic of the operators around the stack without a GPU: scratch planning and refusals that need no context."""
import ctypes

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
