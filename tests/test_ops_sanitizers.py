"""The linear and differential attention's validation layer
(``csrc/sol_api_ops.cpp``, its launchers as host stubs, ``tests/asan/ops_stubs.cpp``)
under AddressSanitizer and UndefinedBehaviorSanitizer: every refusal of
test_ops_abi.py, and one valid call of every entry point (CPU only)."""
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
state = lambda: buf(B * H * D * D * 4)
f = lambda n: buf(4 * n)
q, out = tensor(B, H, N, D), tensor(B, H, N, D)
k, v = tensor(B, Hk, N, D), tensor(B, Hk, N, D)
assert sol.sol_lin_attn_fwd(q, None, k, sol.strides(0, N * D, D), v, None, out, None, f(H), state(), state(), f(B), B, H, Hk,
                            N, D, 1.0, None, 0, None) == 0, sol.sol_last_error()
ws = sol.sol_lin_attn_bwd_workspace_bytes(B, H, Hk, N, D)
s = state()
assert sol.sol_lin_attn_bwd(out, None, q, None, k, None, v, None, tensor(B, H, N, D), None, tensor(B, Hk, N, D), None,
                            tensor(B, Hk, N, D), None, f(H), state(), s, s, f(B), B, H, Hk, N, D, 1.0, buf(ws), ws, None) == 0
assert sol.sol_lin_attn_step(tensor(B, H, D), None, tensor(B, Hk, D), None, tensor(B, Hk, D), None, tensor(B, H, D), None,
                             f(H), buf(3 * H * D * D * 4), f(B), B, H, Hk, 3, D, 1.0, None) == 0
q, k, v = tensor(B, 2 * H, N, D), tensor(B, 2 * Hk, M, D), tensor(B, Hk, M, D)
out2, lse, lam = tensor(B, H, N, 3, D), f(B * 2 * H * N), f(H)
assert sol.sol_diff_attn_fwd(q, None, k, None, v, None, out, None, out2, lse, lam, f(B), f(B), B, H, Hk, 2 * Hk, N, M, D,
                             1.0, 1, None, 0, None) == 0, sol.sol_last_error()
ws = sol.sol_diff_attn_bwd_workspace_bytes(B, H, Hk, N, M, D)
assert sol.sol_diff_attn_bwd(tensor(B, H, N, D), None, q, None, k, None, v, None, out, None, out2, lse, lam,
                             tensor(B, 2 * H, N, D), None, tensor(B, 2 * Hk, M, D), None, tensor(B, Hk, M, D), None, f(H),
                             f(B), f(B), B, H, Hk, 2 * Hk, N, M, D, 1.0, 1, buf(ws), ws, None) == 0, sol.sol_last_error()
"""


def test_validation_layer_under_asan(tmp_path):
    import test_sanitizers as san  # (its builds)
    lib = str(tmp_path / "libsol_ops_asan.so")
    stubs = os.path.join(san.ROOT, "tests", "asan")
    san._run([san._tool("g++"), "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
              "-I", os.path.join(san.ROOT, "include"), "-I", san.CSRC] + san.SAN +
             [os.path.join(san.CSRC, "sol_api.cpp"), os.path.join(san.CSRC, "sol_api_ops.cpp"),
              os.path.join(stubs, "hip_stubs.cpp"), os.path.join(stubs, "ops_stubs.cpp"), "-o", lib])
    code = ("import sys, pytest\n"
            "from paper_2609_35110_amd import sol\n"
            "sol.LIB_PATH = %r\n" % lib + VALID +
            "sys.exit(pytest.main(['tests/test_ops_abi.py', '-q', '-x', '-p', 'no:cacheprovider', '-k', 'refusals']))\n")
    assert " passed" in san._child(code, tmp_path)
