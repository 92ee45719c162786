"""What rotation, windows, accumulated weights and eviction refuse, as far as it shows without a GPU, and the struct that describes a rotation."""
import ast
import ctypes
import os
import re

import torch

from paper_2506_15704_amd import binding as b


def test_calls_without_a_context():
    kv, rot = ctypes.byref(b.lfps_kv()), ctypes.byref(b.lfps_rotary())
    assert b._lib.lfps_rotate_append(None, rot, None, None, None, 0, None, None, 0, kv, None, 0, None) == b.LFPS_EINVAL
    assert b._lib.lfps_window_attn(None, None, 0, None, 0, kv, 1, 0, None, None) == b.LFPS_EINVAL
    assert b._lib.lfps_window_attn_decode(None, None, kv, 1, 0, None, None) == b.LFPS_EINVAL
    assert b._lib.lfps_attn_mass(None, None, 0, None, 0, kv, None, 1.0, None, None) == b.LFPS_EINVAL
    assert b._lib.lfps_full_attn_mass_decode(None, None, kv, None, 1.0, None, None, None) == b.LFPS_EINVAL
    assert b._lib.lfps_evict(None, kv, None, None, 0, 0, None, None, None, None, None) == b.LFPS_EINVAL


def test_the_rotation_mirrors_the_header():
    src = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(b.__file__))), "include", "lfps.h")).read()
    body = re.search(r"typedef struct \{([^}]*)\}\s*lfps_rotary\s*;", re.sub(r"/\*.*?\*/", "", src, flags=re.S)).group(1)
    want = []
    for decl in (d.strip() for d in body.split(";")):
        if decl:
            kind, name = re.match(r"(.+?[\s*])([a-z_]+)$", decl).groups()
            want.append((name, {"float": ctypes.c_float, "int32_t": ctypes.c_int32}.get(kind.strip(), ctypes.c_void_p)))
    assert [tuple(f[:2]) for f in b.lfps_rotary._fields_] == want


def test_kernel_slots_have_names():
    assert b.kernel_names()[-4:] == ["rotate_append", "window_attn", "attn_mass", "evict"]


def test_weights_have_to_be_on_the_gpu():
    try:
        b._ptr(torch.zeros(128), torch.float32, (128,), "q_weight", torch.device("cuda", 0))
    except TypeError as e:
        assert "q_weight" in str(e)
    else:
        raise AssertionError("a host tensor was taken")


def test_the_documented_cache_that_evicts_turns_by_given_positions():
    """After an eviction a token's row is not its place in the text."""
    readme = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(b.__file__))), "README.md")).read()
    evicting = 0
    for block in re.findall(r"```python\n(.*?)```", readme, flags=re.S):
        calls = {n.func.attr: n for n in ast.walk(ast.parse(block)) if isinstance(n, ast.Call) and isinstance(n.func, ast.Attribute)}
        if "lfps_evict" in calls:
            evicting += 1
            positions = calls["lfps_rotate_append"].args[4]
            assert not (isinstance(positions, ast.Constant) and positions.value is None)
    assert evicting
