"""Descriptors of the operators of 8 and 4 bits, on the host (CPU tensors stand for the current
GPU's; nothing is launched): what a call refuses, its descriptor refuses, and what it takes is
described with the sizes and strides that it has."""
import pytest
import torch

BF, F32, I32, U8, E4 = torch.bfloat16, torch.float32, torch.int32, torch.uint8, torch.float8_e4m3fn


@pytest.fixture
def ops(monkeypatch):
    import paper_2608_13499_amd as o
    lib = o._lib
    o.load()

    def current():  # the device number of CPU tensors
        lib._i32, lib._f32, lib._f64 = I32, F32, torch.float64
        return -1
    monkeypatch.setattr(lib, "_current", current)
    for name in ("_i32", "_f32", "_f64"):
        monkeypatch.setattr(lib, name, None)
    return o


def e4(*shape):
    return torch.zeros(*shape, dtype=U8).view(E4)


def refuses(ops, make, good, cases):
    make(**good)
    for bad in cases:
        with pytest.raises(ops.OpscaleError):
            make(**dict(good, **bad))
            pytest.fail(f"taken: { {n: (tuple(t.shape), t.dtype, t.stride()) if torch.is_tensor(t) else t for n, t in bad.items()} }")


def test_quantize(ops):
    x = torch.zeros(6, 256, dtype=BF)
    good = dict(x=x, q=e4(6, 256), scales=torch.zeros(2, 6))
    refuses(ops, ops.desc_quantize_fp8, good, (
        dict(x=torch.zeros(256, 6, dtype=BF).t()), dict(x=torch.zeros(6, 512, dtype=BF)[:, ::2]), dict(x=x.half()), dict(x=x[0]),
        dict(q=e4(5, 256)), dict(q=e4(6, 128)), dict(q=e4(6, 512)[:, :256]), dict(q=torch.zeros(6, 256, dtype=U8)),
        dict(scales=torch.zeros(6, 2).t()), dict(scales=torch.zeros(1, 6)), dict(scales=torch.zeros(2, 6).double())))
    a = ops.desc_quantize_fp8(torch.zeros(6, 512, dtype=BF)[:, :256], *list(good.values())[1:]).u.quantize_fp8
    assert (a.x_row_stride, a.M, a.K) == (512, 6, 256)
    # of a single row any stride is one
    one = torch.zeros(64, dtype=BF).as_strided((1, 16), (4, 1))
    a = ops.desc_quantize_fp8(one, e4(1, 16), torch.zeros(1, 1)).u.quantize_fp8
    assert (a.x_row_stride, a.M, a.K) == (16, 1, 16)


def test_linear(ops):
    M, N, K = 300, 520, 400
    good = dict(x=e4(M, K), x_scales=torch.zeros(4, M), W=e4(N, K), w_scales=torch.zeros(5, 4),
                y=torch.zeros(M, N, dtype=BF), bias=torch.zeros(N, dtype=BF))
    refuses(ops, ops.desc_linear_fp8, good, (
        dict(W=e4(N, K - 16)), dict(W=e4(N, K + 16)), dict(W=e4(N, 2 * K)[:, :K]), dict(W=e4(K, N).t()), dict(W=e4(N - 8, K)),
        dict(W=torch.zeros(N, K, dtype=U8)), dict(x=e4(M, 2 * K)[:, :K]), dict(x=torch.zeros(M, K, dtype=BF)), dict(x=e4(K)),
        dict(x_scales=torch.zeros(3, M)), dict(x_scales=torch.zeros(M, 4).t()), dict(x_scales=torch.zeros(4, M, dtype=BF)),
        dict(w_scales=torch.zeros(4, 4)), dict(w_scales=torch.zeros(4, 5).t()), dict(w_scales=torch.zeros(5, 4).double()),
        dict(y=torch.zeros(M - 1, N, dtype=BF)), dict(y=torch.zeros(M, N + 8, dtype=BF)[:, :N]), dict(y=torch.zeros(M, N)),
        dict(bias=torch.zeros(N)), dict(bias=torch.zeros(N - 8, dtype=BF)), dict(bias=torch.zeros(2 * N, dtype=BF)[::2]),
        dict(workspace=torch.zeros(64, dtype=U8)[::2])))
    a = ops.desc_linear_fp8(**good).u.linear_fp8
    assert (a.M, a.N, a.K, a.bias) == (M, N, K, good["bias"].data_ptr())


def test_linear_workspace(ops):
    """As opscale_linear's descriptor: allocated and kept, given, or none."""
    M, N, K = 256, 512, 4096
    args = e4(M, K), torch.zeros(32, M), e4(N, K), torch.zeros(4, 32), torch.zeros(M, N, dtype=BF)
    need = ops.opscale_linear_fp8_workspace_size(M, N, K)
    d = ops.desc_linear_fp8(*args)
    assert need > 0 and d.u.linear_fp8.workspace_bytes == need and d.u.linear_fp8.workspace == d._keep.data_ptr()
    mine = torch.empty(need + 5, dtype=U8)
    a = ops.desc_linear_fp8(*args, workspace=mine).u.linear_fp8
    assert (a.workspace, a.workspace_bytes) == (mine.data_ptr(), need + 5)
    a = ops.desc_linear_fp8(*args, workspace=False).u.linear_fp8
    assert (a.workspace, a.workspace_bytes) == (None, 0)


def caches(nb=4, Hkv=2, bs=16, D=128):
    return torch.zeros(nb, Hkv, bs, D // 2 + D // 32, dtype=U8)


def test_kv_write(ops):
    kv = torch.zeros(9, 5, 128, dtype=BF)
    good = dict(k=kv[:, :2], v=kv[:, 2:4], k_cache=caches(), v_cache=caches(), slot_mapping=torch.zeros(9, dtype=I32))
    refuses(ops, ops.desc_kv_write_fp4, good, (
        dict(v=kv[:, 2:4].contiguous()), dict(v=kv[:8, 2:4]), dict(v=kv[:, 2:4].float()), dict(k=kv[:, :3], v=kv[:, 2:]),
        dict(k=kv[:, :4:2], v=kv[:, 1::2][:, :2]), dict(k=kv[:, :2, :64], v=kv[:, 2:4, :64]), dict(k=kv.half()[:, :2]),
        dict(k_cache=caches(Hkv=3)), dict(v_cache=caches(nb=3)), dict(v_cache=caches(D=64)), dict(k_cache=caches().view(torch.int8)),
        dict(k_cache=caches(nb=8)[::2]), dict(k_cache=caches()[..., :67]), dict(slot_mapping=torch.zeros(8, dtype=I32)),
        dict(slot_mapping=torch.zeros(9, dtype=torch.int64)), dict(slot_mapping=torch.zeros(18, dtype=I32)[::2])))
    a = ops.desc_kv_write_fp4(**good).u.kv_write_fp4
    assert (a.kv_row_stride, a.T, a.Hkv, a.D, a.block_size, a.num_blocks) == (640, 9, 2, 128, 16, 4)


def test_kv_read(ops):
    kv = torch.zeros(9, 4, 128, dtype=BF)
    good = dict(k_cache=caches(), v_cache=caches(), block_table=torch.zeros(3, 5, dtype=I32),
                cu_seqlens=torch.zeros(4, dtype=I32), k=kv[:, :2], v=kv[:, 2:], first_keys=torch.zeros(3, dtype=I32))
    refuses(ops, ops.desc_kv_read_fp4, good, (
        dict(v=kv[:, 2:].contiguous()), dict(v=kv[:8, 2:]), dict(k=kv[:, :1], v=kv[:, 1:2]), dict(k=kv[:, :2].half()),
        dict(v=kv[:, 2:].float()), dict(v_cache=caches(bs=32)), dict(k_cache=caches(nb=8)[::2]),
        dict(block_table=torch.zeros(15, dtype=I32)), dict(block_table=torch.zeros(5, 3, dtype=I32).t()),
        dict(cu_seqlens=torch.zeros(3, dtype=I32)), dict(cu_seqlens=torch.zeros(4, dtype=torch.int64)),
        dict(first_keys=torch.zeros(2, dtype=I32)), dict(first_keys=torch.zeros(3))))
    a = ops.desc_kv_read_fp4(**good).u.kv_read_fp4
    assert (a.kv_row_stride, a.B, a.total_tokens, a.Hkv, a.D, a.block_size, a.max_blocks_per_seq, a.num_blocks) == \
        (512, 3, 9, 2, 128, 16, 5, 4)


def test_attn_decode(ops):
    q = torch.zeros(3, 8, 128, dtype=BF)
    good = dict(q=q, k_cache=caches(), v_cache=caches(), block_table=torch.zeros(3, 5, dtype=I32),
                context_lens=torch.zeros(3, dtype=I32), out=torch.zeros(3, 8, 128, dtype=BF), max_context_len=80, scale=0.1,
                workspace=torch.zeros(1 << 16, dtype=U8), softcap=3.0, window=7, slopes=torch.zeros(8),
                prefix_lens=torch.zeros(3, dtype=I32), doc_starts=torch.zeros(3, dtype=I32))
    refuses(ops, ops.desc_attn_decode_fp4, good, (
        dict(q=torch.zeros(3, 8, 64, dtype=BF)), dict(q=torch.zeros(3, 8, 256, dtype=BF)[..., ::2]), dict(q=q.half()),
        dict(k_cache=caches(D=64), v_cache=caches(D=64)), dict(v_cache=caches(Hkv=4)), dict(v_cache=caches(nb=8)[::2]),
        dict(block_table=torch.zeros(2, 5, dtype=I32)), dict(block_table=torch.zeros(3, 5)), dict(block_table=torch.zeros(5, 3, dtype=I32).t()),
        dict(context_lens=torch.zeros(2, dtype=I32)), dict(context_lens=torch.zeros(3, dtype=torch.int64)),
        dict(out=torch.zeros(3, 8, 128)), dict(out=torch.zeros(2, 8, 128, dtype=BF)), dict(slopes=torch.zeros(7)),
        dict(slopes=torch.zeros(8, dtype=BF)), dict(prefix_lens=torch.zeros(3)), dict(doc_starts=torch.zeros(4, dtype=I32)),
        dict(window=-1), dict(workspace=torch.zeros(64, dtype=U8)[::2])))
    wide = torch.zeros(3, 10, 128, dtype=BF)
    a = ops.desc_attn_decode_fp4(**dict(good, q=wide[:, :8])).u.attn_decode_fp4
    assert (a.q_row_stride, a.B, a.Hq, a.Hkv, a.D, a.block_size, a.max_blocks_per_seq, a.num_blocks) == (1280, 3, 8, 2, 128, 16, 5, 4)
    assert (a.mods.softcap, a.mods.window, a.mods.slopes) == (3.0, 7, good["slopes"].data_ptr())


def test_tensors_of_another_device(ops, monkeypatch):
    """Host tensors where a GPU is the current device."""
    monkeypatch.setattr(ops._lib, "_current", lambda: 0)
    for name in ("_i32", "_f32"):
        monkeypatch.setattr(ops._lib, name, getattr(torch, {"_i32": "int32", "_f32": "float32"}[name]))
    kv = torch.zeros(9, 4, 128, dtype=BF)
    for make in (lambda: ops.desc_quantize_fp8(torch.zeros(6, 256, dtype=BF), e4(6, 256), torch.zeros(2, 6)),
                 lambda: ops.desc_linear_fp8(e4(4, 128), torch.zeros(1, 4), e4(8, 128), torch.zeros(1, 1), torch.zeros(4, 8)),
                 lambda: ops.desc_kv_write_fp4(kv[:, :2], kv[:, 2:], caches(), caches(), torch.zeros(9, dtype=I32))):
        with pytest.raises(ops.OpscaleError):
            make()
