"""What the calls around the 8-bit cache and the log probabilities refuse before any CUDA call (no GPU needed)."""
import ctypes as C
import importlib


def test_missing_arguments():
    B = importlib.import_module("paper_2509_18362_b200.binding")
    kv, none, some = B.fmtp_kv8(), None, 4096
    assert B.lib.fastmtp_kv8_append(none, some, some, 128, C.byref(kv), 1, 1, none, none, none) == -1
    assert B.lib.fastmtp_kv8_read(none, C.byref(kv), 1, 1, none, none, some, some, none, none) == -1
    assert B.lib.fastmtp_kv8_attention(none, some, 128, C.byref(kv), 1, 1, none, some, none, none) == -1
    assert B.lib.fastmtp_logprobs(none, some, 0, 128, some, 1, 128, some, none, 0, none, none, none, none) == -1
