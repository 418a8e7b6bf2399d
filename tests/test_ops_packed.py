"""Tensors side by side in one buffer, without a GPU: rows that meet are refused,
rows that only share a span are not (checked with the launchers as host stubs)."""
import os

CODE = r"""
import ctypes, itertools, random
from paper_2609_35110_amd import sol
sol.LIB_PATH = %r
D = 128
L = sol.lib()
room = ctypes.create_string_buffer(1 << 22)
base = (ctypes.addressof(room) + 4095) // 4096 * 4096
apart = ctypes.create_string_buffer(1 << 20)
other = (ctypes.addressof(apart) + 4095) // 4096 * 4096
S = sol.strides

def step_like(rows_q, out_at, out_st, B, H, N):
    # q at `base` with its strides, out where asked; k and v elsewhere
    st = sol.sol_lin_attn_fwd(base, S(*rows_q), other, S(0, 0, 0), other, S(0, 0, 0), base + 2 * out_at, S(*out_st), other, None,
                              None, None, B, H, H, N, D, 1.0, None, 0, None)
    return st, sol.sol_last_error()

def rows(at, st, B, H, N):
    return {at + b * st[0] + h * st[1] + n * st[2] for b in range(B) for h in range(H) for n in range(N)}

def meets(a, b):
    return any(abs(x - y) < D for x in a for y in b)

# known layouts: [B][N][3][H][D], [B][3][H][N][D], [B][H][N][3][D], [B][N][H][3][D]
B, H, N = 2, 3, 4
for name, st, part in (("bn3hd", (N * 3 * H * D, D, 3 * H * D), H * D), ("b3hnd", (3 * H * N * D, N * D, D), H * N * D),
                       ("bhn3d", (H * N * 3 * D, N * 3 * D, 3 * D), D), ("bnh3d", (N * H * 3 * D, 3 * D, H * 3 * D), D)):
    for i in (1, 2):
        st_, err = step_like(st, i * part, st, B, H, N)
        assert st_ == 0, (name, i, err)
    for off in (0, 8, part - 8, part + 8 - part %% 16):
        got, err = step_like(st, off, st, B, H, N)
        if meets(rows(0, st, B, H, N), rows(off, st, B, H, N)):
            assert got == -1 and "overlaps" in err, (name, off, got)

# any strides: what is taken never meets
rng = random.Random(1)
taken = refused = 0
for _ in range(4000):
    B, H, N = (rng.choice([1, 2, 3]) for _ in range(3))
    dims = [B, H, N]
    def strides():
        order = rng.sample(range(3), 3)
        st, at = [0, 0, 0], D
        for i in order:
            st[i] = at + 8 * rng.choice([0, 0, 16, 16, 32, 48, 3])
            at = st[i] * dims[i]
        return tuple(st)
    a, b = strides(), strides()
    if rng.random() < 0.7:
        b = a
    off = 8 * rng.randrange(0, 160)
    got, err = step_like(a, off, b, B, H, N)
    real = meets(rows(0, a, B, H, N), rows(off, b, B, H, N))
    assert got in (0, -1), (got, err)
    if got == 0:
        assert not real, (a, b, off, dims)
        taken += 1
    else:
        refused += 1
print("taken", taken, "refused", refused)
assert taken > 100 and refused > 1000
print("1 passed")
"""


def test_only_rows_that_meet_are_refused(tmp_path):
    import test_sanitizers as san  # (its builds)
    lib = str(tmp_path / "libsol_packed.so")
    stubs = os.path.join(san.ROOT, "tests", "asan")
    san._run([san._tool("g++"), "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
              "-I", os.path.join(san.ROOT, "include"), "-I", san.CSRC] + san.SAN +
             [os.path.join(san.CSRC, "sol_api.cpp"), os.path.join(san.CSRC, "sol_api_ops.cpp"),
              os.path.join(stubs, "hip_stubs.cpp"), os.path.join(stubs, "ops_stubs.cpp"), "-o", lib])
    assert "1 passed" in san._child(CODE % lib, tmp_path)
