"""The validation layer of the norm and rotation at given positions and of cross
attention (``csrc/sol_api_cross.cpp``, its launchers as host stubs,
``tests/asan/cross_stubs.cpp``) under AddressSanitizer and
UndefinedBehaviorSanitizer: every refusal of test_cross_abi.py, and valid calls of
every entry point (CPU only)."""
import os

VALID = """
import ctypes
from paper_2609_35110_amd import sol
keep = []
def buf(n):
    b = ctypes.create_string_buffer(n + 64)
    keep.append(b)
    return (ctypes.addressof(b) + 15) // 16 * 16
def tensor(*shape):
    n = 2
    for s in shape:
        n *= s
    return buf(n)
B, H, Hk, N, M, D = 2, 4, 2, 5, 7, 128
f = lambda n: buf(4 * n)
q, k, pos, tab, g = tensor(B, H, N, D), tensor(B, Hk, N, D), f(3 * N), f(4096), f(D)
for kk, gg in ((k, g), (None, None)):  # with k and without, where its pointers are not looked at
    h = Hk if kk else 0
    for out in (tensor(B, H, N, D), q):
        assert sol.sol_qk_norm_rope(q, None, kk, None, out, None, kk and tensor(B, Hk, N, D), None, g, gg, 1e-6, pos, 0, tab,
                                    2, 3, 4, 32, 48, 48, f(B), B, H, h, N, D, None) == 0, sol.sol_last_error()
    ws = sol.sol_qk_norm_rope_bwd_workspace_bytes(B, H, h, N, D)
    assert sol.sol_qk_norm_rope_bwd(tensor(B, H, N, D), None, kk and tensor(B, Hk, N, D), None, q, None, kk, None,
                                    tensor(B, H, N, D), None, kk and tensor(B, Hk, N, D), None, g, gg, f(D), gg and f(D),
                                    1e-6, pos, 0, tab, 2, 3, 4, 32, 48, 48, f(B), B, H, h, N, D, buf(ws), ws,
                                    None) == 0, sol.sol_last_error()
# no norm, no positions: q and the table are not looked at
assert sol.sol_qk_norm_rope_bwd(out, None, None, None, None, None, None, None, tensor(B, H, N, D), None, None, None, None,
                                None, None, None, 0.0, None, 0, None, 0, 0, 0, 32, 48, 48, None, B, H, 0, N, D, None, 0,
                                None) == 0, sol.sol_last_error()
k, v = tensor(Hk, M, D), tensor(Hk, M, D)
st = sol.strides(0, M * D, D)
out, left, lse = tensor(B, H, N, D), tensor(B, H, N, D), f(B * H * N)
for train in (False, True):
    for mask in (None, buf(B * M) + 1):
        assert sol.sol_cross_attn_fwd(q, None, k, st, v, st, out, None, left if train else None, lse if train else None,
                                      f(B), f(B), mask, B, H, Hk, N, M, D, 0.1, None, 0, None) == 0, sol.sol_last_error()
ws = sol.sol_cross_attn_bwd_workspace_bytes(B, H, Hk, N, M, D, 1)
assert sol.sol_cross_attn_bwd(tensor(B, H, N, D), None, q, None, k, st, v, st, out, None, left, lse, tensor(B, H, N, D), None,
                              tensor(B, Hk, M, D), None, tensor(B, Hk, M, D), None, f(B), f(B), buf(B * M), B, H, Hk, N, M,
                              D, 0.1, buf(ws), ws, None) == 0, sol.sol_last_error()
M = 1100
k, v = tensor(B, Hk, M, D), tensor(B, Hk, M, D)
ws = sol.sol_cross_attn_fwd_workspace_bytes(B, H, Hk, N, M, D, 0)
assert sol.sol_cross_attn_fwd(q, None, k, None, v, None, out, None, None, None, None, None, None, B, H, Hk, N, M, D, 0.1,
                              buf(ws), ws, None) == 0, sol.sol_last_error()
"""


def test_validation_layer_under_asan(tmp_path):
    import test_sanitizers as san  # (its builds)
    lib = str(tmp_path / "libsol_cross_asan.so")
    stubs = os.path.join(san.ROOT, "tests", "asan")
    san._run([san._tool("g++"), "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
              "-I", os.path.join(san.ROOT, "include"), "-I", san.CSRC] + san.SAN +
             [os.path.join(san.CSRC, "sol_api.cpp"), os.path.join(san.CSRC, "sol_api_cross.cpp"),
              os.path.join(stubs, "hip_stubs.cpp"), os.path.join(stubs, "cross_stubs.cpp"), "-o", lib])
    code = ("import sys, pytest\n"
            "from paper_2609_35110_amd import sol\n"
            "sol.LIB_PATH = %r\n" % lib + VALID +
            "sys.exit(pytest.main(['tests/test_cross_abi.py', '-q', '-x', '-p', 'no:cacheprovider', '-k', 'refusals']))\n")
    assert " passed" in san._child(code, tmp_path)
