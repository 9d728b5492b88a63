"""The refusals of the attention level's operators (no GPU): every call here
is wrong, or is on the CPU, and raises before anything is launched."""
import pytest
import torch

from paper_2008_06967_amd import ops

T = torch.zeros


def test_cpu_tensors_are_refused():
    p = ops.Int8Params(T((4, 8), dtype=torch.int8), torch.ones(4), device="cpu")
    r = ops.RotaryParams([2, 2], device="cpu")
    q = T(1, 3, 2, 8)
    for f in (lambda: ops.group_norm(T(1, 5, 8), 2), lambda: ops.quantize_int8(T(3, 8)),
              lambda: ops.linear_int8(T(3, 8), p), lambda: ops.rotary(q, T(1, 3, 2), r),
              lambda: ops.cross_attention(q, q, q)):
        with pytest.raises(ValueError, match="GPU"):
            f()


def test_group_norm_refusals():
    x = T(2, 5, 8)
    for kw in (dict(act="tanh"), dict(gamma=torch.ones(7)), dict(gamma=torch.ones(8, dtype=torch.float64)),
               dict(beta=torch.ones(16)[::2]), dict(lens=T(2)), dict(lens=T(3, dtype=torch.int32)),
               dict(out=T(2, 5, 9))):
        with pytest.raises(ValueError):
            ops.group_norm(x, 2, **kw)
    for bad in (T(5, 8), T(2, 5, 8, dtype=torch.float16), T(2, 8, 5).transpose(1, 2), T(2, 10, 8)[:, ::2][:, :3]):
        with pytest.raises(ValueError):
            ops.group_norm(bad, 2)


def test_linear_refusals():
    p = ops.Int8Params(T((4, 8), dtype=torch.int8), torch.ones(4), torch.ones(4), device="cpu")
    assert p.W.stride(0) == 16 and p.ld == 16
    q = ops.int8_rows(T((3, 8), dtype=torch.int8))
    for args, kw in (((T(3, 7), p), {}), ((T(3, 8, dtype=torch.float16), p), {}), ((q, p), {}),
                     ((T(3, 8), p), dict(x_scale=torch.ones(3))), ((q, p), dict(x_scale=torch.ones(4))),
                     ((T(3, 8), p), dict(out=T(3, 5))), ((T(3, 8), p), dict(out=T(3, 4), out_dtype=torch.bfloat16)),
                     ((T(3, 8), p), dict(out_dtype=torch.float16))):
        with pytest.raises(ValueError):
            ops.linear_int8(*args, **kw)
    for args in ((T(4, 8), torch.ones(4)), (T((4, 8), dtype=torch.int8), torch.ones(5)),
                 (T((4, 8), dtype=torch.int8), torch.ones(4), torch.ones(3)), (T(8, dtype=torch.int8), torch.ones(8))):
        with pytest.raises(ValueError):
            ops.Int8Params(*args, device="cpu")
    with pytest.raises(ValueError):
        ops.int8_rows(T(3, 8))
    # 16-byte rows that end with their storage, behind the last row's start
    with pytest.raises(ValueError, match="padding"):
        ops.linear_int8(T(16 * 2 + 8, dtype=torch.int8).as_strided((3, 8), (16, 1)), p, x_scale=torch.ones(3))


def test_int8_rows_layout():
    q = torch.arange(-15, 15, dtype=torch.int8).view(2, 3, 5)
    t = ops.int8_rows(q)
    assert torch.equal(t, q) and t.stride() == (48, 16, 1)
    assert bool((t.as_strided((6, 16), (16, 1))[:, 5:] == 0).all())


def test_rotary_refusals():
    x, pos = T(3, 2, 8), T(3, 2)
    p = ops.RotaryParams([2, 2], device="cpu")
    for args, kw in (((T(8), pos, p), {}), ((x, T(3, 3), p), {}), ((x, T(4, 2), p), {}), ((x, pos.double(), p), {}),
                     ((x, pos, p), dict(out=T(3, 2, 9))), ((x, pos, p), dict(out=T(3, 2, 8, dtype=torch.bfloat16))),
                     ((T(3, 8, 2).transpose(1, 2), pos, p), {}), ((T(3, 4, 8)[:, ::2], pos, p), {})):
        with pytest.raises(ValueError):
            ops.rotary(*args, **kw)
    for sec in ([], [1, 1, 1, 1, 1], [3, -1]):
        with pytest.raises(ValueError):
            ops.RotaryParams(sec, device="cpu")
    with pytest.raises(ValueError):
        ops.RotaryParams([2, 2], freq=torch.ones(3), device="cpu")


def test_rotary_frequencies():
    p = ops.RotaryParams([2, 0, 3], base=100.0, scale=2.0, device="cpu")
    want = [2.0, 2.0 / 10.0] + [2.0 * 100.0 ** (-i / 3) for i in range(3)]
    assert torch.equal(p.freq, torch.tensor(want, dtype=torch.float32))


def test_cross_attention_refusals():
    q, k = T(2, 5, 4, 8), T(2, 7, 2, 8)
    ok = dict(k_len=T(2, dtype=torch.int32), k_mask=T((2, 7), dtype=torch.bool))
    for args, kw in (((q[0], k, k), {}), ((q, k, k[:, :6]), {}), ((q, k[:1], k[:1]), {}), ((q, k[..., :7], k[..., :7]), {}),
                     ((q, k.bfloat16(), k.bfloat16()), {}), ((q.half(), k.half(), k.half()), {}),
                     ((q, k, k), dict(k_len=T(2))), ((q, k, k), dict(k_len=T(3, dtype=torch.int32))),
                     ((q, k, k), dict(k_mask=T(2, 7))), ((q, k, k), dict(k_mask=T((2, 8), dtype=torch.bool))),
                     ((q, k, k), dict(ok, out=T(2, 5, 4, 9))), ((q, k, k), dict(out=T(2, 5, 4, 8).bfloat16())),
                     ((T(2, 5, 8, 4).transpose(2, 3), k, k), {})):
        with pytest.raises(ValueError):
            ops.cross_attention(*args, **kw)


def test_out_must_not_be_an_input():
    x = torch.zeros(2, 8, 16)
    with pytest.raises(ValueError, match="out must not be an input"):
        ops.group_norm(x, 4, out=x)
    with pytest.raises(ValueError, match="out must not be an input"):
        ops.group_norm(x[:, :, :8], 4, out=x[:, :, :8])
    q = torch.zeros(1, 8, 2, 16)
    k, v = torch.zeros(1, 8, 2, 16), torch.zeros(1, 8, 2, 16)
    for o in (q, k, v):
        with pytest.raises(ValueError, match="out must not be an input"):
            ops.cross_attention(q, k, v, out=o)
    # other columns of one buffer are apart: the call goes on to the device check
    with pytest.raises(ValueError, match="must be on a GPU"):
        ops.group_norm(x[..., :8], 4, out=x[..., 8:])


def test_import_without_gpu_functions():
    """The module loads, and refuses CPU tensors, on a torch that lacks the
    GPU build's functions."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = ("import torch\n"
            "for n in ('_cuda_getDevice', '_cuda_getCurrentRawStream'):\n"
            "    if hasattr(torch._C, n): delattr(torch._C, n)\n"
            "from paper_2008_06967_amd import ops\n"
            "try:\n"
            "    ops.group_norm(torch.zeros(1, 5, 8), 2)\n"
            "except ValueError as e:\n"
            "    assert 'GPU' in str(e)\n"
            "    print('refused')\n")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=root)
    assert r.returncode == 0 and "refused" in r.stdout, r.stderr[-2000:]
