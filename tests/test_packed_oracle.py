"""Pins of the packed-batch oracle, and the refusals of the packed entry points (host checks: no device needed)."""
import ctypes
import os

import numpy as np
import pytest

from oracle import hyb_oracle as O
from oracle import packed_oracle as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2602_21760_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.lib()


def test_layout_counts_and_order():
    offsets, request, positions = P.packed_layout([(1, 2, 3, 2), (0, 5, 5, 0), (2, 1, 2, 1)], 100, True)
    assert offsets.tolist() == [0, 8, 8, 13]
    assert request.tolist() == [0] * 8 + [2] * 5
    assert positions.tolist() == [[0, 0, 0], [0, 0, 1], [0, 0, 2], [0, 1, 0], [0, 1, 1], [0, 1, 2], [3, 3, 3], [4, 4, 4],
                                  [0, 0, 0], [0, 0, 1], [1, 0, 0], [1, 0, 1], [2, 2, 2]]
    offsets, request, _ = P.packed_layout([(1, 2, 3, 2), (-1, 5, 5, 1), (2, 1, 2, 1)], 10)
    assert offsets.tolist() == [0, 8, 9, 10] and request.tolist() == [0] * 8 + [1, 2]


@pytest.mark.parametrize("halves", [False, True])
def test_rotary_properties(halves):
    rng = np.random.default_rng(1)
    dims, pos = (8, 12, 12), rng.integers(-50, 1000, (7, 3))
    x, y = rng.standard_normal((2, 7, 3, 48))
    r = P.rotary(x, pos, dims, halves=halves)
    np.testing.assert_allclose(P.rotary(r, pos, dims, halves=halves, inverse=True), x, atol=1e-12)                 # a rotation
    np.testing.assert_allclose(np.linalg.norm(r, axis=2), np.linalg.norm(x, axis=2))
    np.testing.assert_array_equal(r[..., 32:], x[..., 32:])
    np.testing.assert_allclose((r * y).sum(), (x * P.rotary(y, pos, dims, halves=halves, inverse=True)).sum())      # inverse = transpose
    # products of queries and keys depend on the difference of positions only
    a = (P.rotary(x, pos, dims, halves=halves) * P.rotary(y, pos + 5, dims, halves=halves)).sum(2)
    b = (P.rotary(x, pos + 77, dims, halves=halves) * P.rotary(y, pos + 82, dims, halves=halves)).sum(2)
    np.testing.assert_allclose(a, b, atol=1e-10)


def test_packed_attention_is_attention_per_sequence():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((9, 4, 64)), rng.standard_normal((11, 2, 64)), rng.standard_normal((11, 2, 64))
    got = P.packed_attention(q, k, v, [0, 4, 4, 9], [0, 6, 6, 11])
    for (q0, q1), (k0, k1) in (((0, 4), (0, 6)), ((4, 9), (6, 11))):
        rep = lambda x: np.repeat(x[k0:k1], 2, axis=1).transpose(1, 0, 2)[None]      # noqa: E731
        ref = O.attention(q[q0:q1].transpose(1, 0, 2)[None], rep(k), rep(v))
        np.testing.assert_allclose(got[q0:q1].reshape(1, q1 - q0, -1), ref, atol=1e-12)
    got = P.packed_attention(q, k, v, [0, 9], [0, 3], causal=True)                    # six queries see nothing, the seventh one key
    assert not got[:6].any()
    np.testing.assert_allclose(got[6, 3], v[0, 1])


def _rotary_desc(binding, **changes):
    f = dict(tokens=4, q_heads=2, k_heads=2, head_dim=64, axes=2, axis_dims=(32, 32), axis_scale=(), theta=10000.0, pairs=0, inverse=0, q_scale=1.0, dtype=1,
             q_stride=128, k_stride=128, q_out_stride=128, k_out_stride=128)
    f.update(changes)
    d = binding.RotaryDesc()
    for n, x in f.items():
        if isinstance(x, tuple):
            for i, e in enumerate(x):
                getattr(d, n)[i] = e
        else:
            setattr(d, n, x)
    return d


@pytest.mark.parametrize("changes,code", [
    (dict(tokens=-1), 2), (dict(q_heads=-1), 2), (dict(q_heads=513), 2), (dict(head_dim=72), 2), (dict(head_dim=272), 2), (dict(head_dim=0), 2), (dict(axes=0), 2), (dict(axes=5), 2),
    (dict(axis_dims=(31, 33)), 2), (dict(axis_dims=(0, 64)), 2), (dict(axis_dims=(64, 2)), 2), (dict(axis_dims=(-2, 64)), 2), (dict(pairs=1, axis_dims=(20, 20)), 2), (dict(pairs=2), 3),
    (dict(theta=0.0), 2), (dict(theta=float("nan")), 2), (dict(axis_scale=(float("inf"), 1.0)), 2), (dict(q_scale=float("nan")), 2), (dict(dtype=2), 3),
    (dict(q_stride=120), 2), (dict(k_stride=132), 4), (dict(k_out_stride=64), 2), (dict(q_stride=1 << 31), 2)])
def test_rotary_refusals(lib, changes, code):
    from paper_2602_21760_amd import binding
    d = _rotary_desc(binding, **changes)
    assert lib.hyb_rotary(ctypes.byref(d), 4096, 4096, 8192, 4096, 8192, None) == code, lib.hyb_last_error_string()


def test_rotary_pointer_refusals_and_no_ops(lib):
    from paper_2602_21760_amd import binding
    d = _rotary_desc(binding)
    call = lambda *a: lib.hyb_rotary(ctypes.byref(d), *a, None)      # noqa: E731
    assert lib.hyb_rotary(None, 4096, 4096, 4096, 4096, 4096, None) == 1
    assert call(None, 4096, 4096, 4096, 4096) == 1 and call(4096, None, 4096, 4096, 4096) == 1 and call(4096, 4096, 4096, 4096, None) == 1
    assert call(4100, 4096, 4096, 4096, 4096) == 4 and call(4096, 4096, 4104, 4096, 4096) == 4
    d = _rotary_desc(binding, q_out_stride=256)
    assert call(4096, 4096, 4096, 4096, 4096) == 2                    # in place with another stride
    for zero in (dict(tokens=0), dict(q_heads=0, k_heads=0)):
        d = _rotary_desc(binding, **zero)
        assert call(None, None, None, None, None) == 0


def test_layout_refusals(lib):
    call = lib.hyb_packed_layout
    assert call(4096, -1, 5, 0, 4096, None, None, None) == 2 and call(4096, 2, -5, 0, 4096, None, None, None) == 2
    assert call(None, 2, 5, 0, 4096, None, None, None) == 1 and call(4096, 2, 5, 0, None, None, None, None) == 1
    assert call(4104, 2, 5, 0, 4096, None, None, None) == 4 and call(4096, 2, 5, 0, 4100, None, None, None) == 4
    assert call(4096, 2, 5, 0, 4096, 4100, None, None) == 4 and call(4096, 2, 5, 0, 4096, None, 4100, None) == 4


def _attention_desc(binding, **changes):
    f = dict(sequences=2, total_q=100, total_k=120, max_q=0, max_k=0, q_heads=4, k_heads=2, head_dim=64, scale=0.0, causal=0, prescaled=0, dtype=1,
             q_token_stride=256, q_head_stride=64, k_token_stride=128, k_head_stride=64, v_token_stride=128, v_head_stride=64, o_token_stride=256, o_head_stride=64)
    f.update(changes)
    return binding.PackedAttentionDesc(**f)


@pytest.mark.parametrize("changes,code", [
    (dict(sequences=-1), 2), (dict(total_q=-1), 2), (dict(total_k=-1), 2), (dict(max_k=-1), 2), (dict(head_dim=32), 2), (dict(head_dim=96), 2), (dict(q_heads=3), 2), (dict(k_heads=0), 2),
    (dict(q_heads=0), 2), (dict(dtype=5), 3), (dict(q_token_stride=260), 4), (dict(v_head_stride=60), 4), (dict(k_token_stride=1 << 23), 2), (dict(k_head_stride=1 << 40), 2),
    (dict(o_token_stride=192), 2), (dict(o_head_stride=56), 2), (dict(total_q=0x7fffffff), 2), (dict(total_k=(1 << 30) + 1), 2), (dict(q_heads=65536 * 2, k_heads=2), 2)])
def test_attention_refusals(lib, changes, code):
    from paper_2602_21760_amd import binding
    d = _attention_desc(binding, **changes)
    assert lib.hyb_packed_attention(ctypes.byref(d), 4096, 4096, 4096, 4096, 4096, 4096, None, 0, None) == code, lib.hyb_last_error_string()


def test_attention_pointer_refusals_workspace_and_no_ops(lib):
    from paper_2602_21760_amd import binding
    d = _attention_desc(binding)
    assert lib.hyb_packed_attention_workspace_bytes(ctypes.byref(d)) == 0 and lib.hyb_packed_attention_workspace_bytes(None) == 0
    assert lib.hyb_packed_attention(None, *[4096] * 6, None, 0, None) == 1
    for i in range(6):
        for bad, code in ((None, 1), (4104, 4)):
            args = [4096] * 6
            args[i] = bad
            assert lib.hyb_packed_attention(ctypes.byref(d), *args, None, 0, None) == code, i
    for zero in (dict(sequences=0), dict(total_q=0)):
        d = _attention_desc(binding, **zero)
        assert lib.hyb_packed_attention(ctypes.byref(d), *[None] * 6, None, 0, None) == 0
    d = _attention_desc(binding, total_q=2, total_k=50000, max_q=1, max_k=40000)      # few rows, many keys: cut
    need = lib.hyb_packed_attention_workspace_bytes(ctypes.byref(d))
    assert need > 0 and need % 256 == 0
    assert lib.hyb_packed_attention(ctypes.byref(d), *[4096] * 6, None, 0, None) == 1
    assert lib.hyb_packed_attention(ctypes.byref(d), *[4096] * 6, 4096, need - 1, None) == 5
    assert lib.hyb_packed_attention(ctypes.byref(d), *[4096] * 6, 4104, need, None) == 4


def test_struct_layouts_match_the_header(tmp_path):
    import shutil
    import subprocess
    from paper_2602_21760_amd import binding
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    structs = {"hyb_rotary_desc": binding.RotaryDesc, "hyb_packed_attention_desc": binding.PackedAttentionDesc}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "hyb.h"', 'int main(void) {']
    for cname, ct in structs.items():
        lines.append('printf("%s size %%zu\\n", sizeof(%s));' % (cname, cname))
        lines += ['printf("%s %s %%zu\\n", offsetof(%s, %s));' % (cname, f, cname, f) for f, _ in ct._fields_]
    (tmp_path / "layout.c").write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(tmp_path / "layout.c"), "-o", str(tmp_path / "layout")], check=True)
    out = subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.split("\n")
    got = {tuple(x.split()[:2]): int(x.split()[2]) for x in out if x}
    for cname, ct in structs.items():
        assert got[(cname, "size")] == ctypes.sizeof(ct)
        for f, _ in ct._fields_:
            assert got[(cname, f)] == getattr(ct, f).offset, (cname, f)


def test_descriptors_from_tensors():
    """Strides, sizes and refusals of the descriptor makers (CPU tensors: nothing is launched)."""
    import torch
    from paper_2602_21760_amd import binding as hb
    qkv = torch.zeros(10, 8, 64, dtype=torch.bfloat16)
    q, k, v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    d = hb.rotary_desc(q, k, (16, 24, 24), axis_scale=(1.0, 0.5, 0.5), q_out=torch.zeros(10, 4, 64, dtype=torch.bfloat16))
    assert (d.tokens, d.q_heads, d.k_heads, d.head_dim, d.axes) == (10, 4, 2, 64, 3) and list(d.axis_dims) == [16, 24, 24, 0]
    assert (d.q_stride, d.q_out_stride, d.k_stride, d.k_out_stride) == (512, 256, 512, 512) and list(d.axis_scale)[:3] == [1.0, 0.5, 0.5]
    assert hb.rotary_desc(q, None, (64,)).k_heads == 0
    for bad in (dict(axis_dims=()), dict(axis_dims=(16,) * 5), dict(axis_dims=(64,), axis_scale=(1.0, 2.0)), dict(axis_dims=(64,), q_scale=0.0), dict(axis_dims=(64,), k_out=q),
                dict(axis_dims=(64,), q_out=q.float())):
        with pytest.raises(ValueError):
            hb.rotary_desc(q, k, **bad)
    with pytest.raises(ValueError):
        hb.rotary_desc(qkv[:, ::2], k, (64,))                         # heads not adjacent
    o = torch.zeros(4, 10, 64, dtype=torch.bfloat16).transpose(0, 1)     # head-major
    cu = torch.tensor([0, 4, 10], dtype=torch.int32)
    d = hb.packed_attention_desc(q, k, v, o, cu, max_k=6, causal=True)
    assert (d.sequences, d.total_q, d.total_k, d.max_k, d.q_heads, d.k_heads, d.head_dim, d.causal) == (2, 10, 10, 6, 4, 2, 64, 1)
    assert (d.q_token_stride, d.q_head_stride, d.o_token_stride, d.o_head_stride, d.v_token_stride) == (512, 64, 64, 640, 512)
    for bad in (lambda: hb.packed_attention_desc(q, k, v[:9], o, cu), lambda: hb.packed_attention_desc(q, k, v, o[:, :2], cu), lambda: hb.packed_attention_desc(q, k[..., :32], v[..., :32], o, cu),
                lambda: hb.packed_attention_desc(q, k, v, o, cu[None]), lambda: hb.packed_attention_desc(q[0], k, v, o[0], cu), lambda: hb.packed_attention_desc(q.transpose(1, 2), k, v, o, cu)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        hb.packed_attention_desc(q, k.float(), v, o, cu)
    one = torch.zeros(1, 4, 64).expand(1, 4, 64)
    assert hb._head_strides(one, "q") == (256, 64) and hb._head_strides(torch.zeros(5, 64)[:, None], "q") == (64, 64)


def test_one_row_of_a_head_major_tensor(lib):
    """The first step over an empty cache: heads far apart, one token, whose stride says nothing."""
    import torch
    from paper_2602_21760_amd import binding as hb
    cache = torch.zeros(8, 8192, 128, dtype=torch.bfloat16)
    cu = torch.tensor([0, 1], dtype=torch.int32)
    for rows in (1, 2):
        k = cache[:, :rows].transpose(0, 1)
        d = hb.packed_attention_desc(k, k, k, k, cu)
        assert (d.k_token_stride, d.k_head_stride) == (1024 if rows == 1 else 128, 8192 * 128)
        # (the strides are accepted: what is missing is the first tensor)
        assert lib.hyb_packed_attention(ctypes.byref(d), None, 4096, 4096, 4096, 4096, 4096, None, 0, None) == 1, lib.hyb_last_error_string()


@pytest.mark.parametrize("scale,code", [(float("nan"), 2), (float("inf"), 2), (3e38, 2), (2e38, 1), (1e-38, 1), (0.0, 1), (-1.0, 1), (float("-inf"), 1)])
def test_attention_scale(lib, scale, code):
    """A scale that is no number is refused, not taken for the default (accepted ones get as far as the missing tensor); one that is not used may be anything."""
    from paper_2602_21760_amd import binding
    call = lambda d: lib.hyb_packed_attention(ctypes.byref(d), None, 4096, 4096, 4096, 4096, 4096, None, 0, None)      # noqa: E731
    assert call(_attention_desc(binding, scale=scale)) == code, lib.hyb_last_error_string()
    assert call(_attention_desc(binding, scale=scale, prescaled=1)) == 1
