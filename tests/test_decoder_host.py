"""CPU-only refusals and sizes of the 4-bit decoder operators (every error is raised by host-side checks, before a device is touched)."""
import ctypes as C

import pytest

import paper_2512_04677_amd as lvx

P, ODD = C.c_void_p(4096), C.c_void_p(4100)


def handle(**kw):
    d = dict(n_layers=2, n_seqs=3, n_kv_heads=4, head_dim=128, max_keys=1000)
    d.update(kw)
    desc, h = lvx.kv4_desc(**d), C.c_void_p()
    assert lvx.load().lvx_kv4_init(C.byref(desc), P, 1 << 60, C.byref(h)) == 0
    return h


def test_norm_refusals():
    f = lvx.load().lvx_rmsnorm_residual
    ok = dict(x=P, ldx=64, r=P, ldr=64, f32=0, g=P, eps=1e-6, n=0, d=64, s=P, lds=64, y=P, ldy=64)

    def status(**kw):
        return f(*{**ok, **kw}.values(), None)

    assert status() == 0                                   # no tokens: nothing to do
    assert status(x=None, r=None, s=None) == 1 and status(r=None) == 1 and status(y=None) == 1
    assert status(x=ODD) == 1 and status(r=ODD) == 1 and status(g=ODD) == 1 and status(s=ODD) == 1 and status(y=ODD) == 1
    assert status(f32=2) == 1 and status(eps=-1.0) == 1 and status(eps=float("nan")) == 1
    assert status(d=60) == 2 and status(d=0) == 2 and status(d=16392, ldx=1 << 15, ldr=1 << 15, lds=1 << 15, ldy=1 << 15) == 2
    assert status(n=-1) == 2 and status(n=1 << 22) == 2 and status(ldx=56) == 2 and status(ldr=68) == 2 and status(lds=56) == 2 and status(ldy=56) == 2
    assert status(r=None, s=None, ldr=0, lds=0) == 0
    g = lvx.load().lvx_rmsnorm_residual_fp8
    assert g(P, 72, P, 72, 0, P, 1e-6, 0, 72, P, 72, P, 80, P, None) == 2          # d % 16
    assert g(P, 64, P, 64, 0, P, 1e-6, 0, 64, P, 64, P, 72, P, None) == 2          # ldq % 16
    assert g(P, 64, P, 64, 0, P, 1e-6, 0, 64, P, 64, P, 64, None, None) == 1       # no row scales
    assert g(P, 64, P, 64, 0, P, 1e-6, 0, 64, P, 64, P, 64, P, None) == 0


def test_quantize_and_linear_refusals():
    lib = lvx.load()
    q = lib.lvx_fp4_quantize
    assert q(P, 64, 0, 64, P, 32, P, 2, None) == 0
    assert q(None, 64, 4, 64, P, 32, P, 2, None) == 1 and q(P, 64, 4, 64, ODD, 32, P, 2, None) == 1 and q(P, 64, 4, 64, P, 32, None, 2, None) == 1
    assert q(P, 64, 4, 48, P, 32, P, 2, None) == 2 and q(P, 56, 4, 64, P, 32, P, 2, None) == 2 and q(P, 64, 4, 64, P, 40, P, 2, None) == 2
    assert q(P, 64, 4, 64, P, 16, P, 2, None) == 2 and q(P, 64, 4, 64, P, 32, P, 1, None) == 2 and q(P, 64, -1, 64, P, 32, P, 2, None) == 2
    ok = dict(a=P, lda=64, w=P, ldw=32, s=P, lds=2, c=P, ldc=16, M=0, N=16, K=64, epi=0, r=None, ldr=0, gate=None)

    def status(f=lib.lvx_linear_fp4, **kw):
        return f(*{**ok, **kw}.values(), None)

    assert status() == 0 and status(epi=lvx.EPI_STORE_F32) == 0
    assert status(a=None) == 1 and status(a=ODD) == 1 and status(w=ODD) == 1 and status(c=ODD) == 1 and status(s=None) == 1
    assert status(K=48) == 2 and status(N=12) == 2 and status(M=-1) == 2 and status(lda=56) == 2 and status(lda=68) == 2
    assert status(ldw=16) == 2 and status(ldw=40) == 2 and status(lds=1) == 2 and status(ldc=8) == 2 and status(ldc=20) == 2
    assert status(epi=4) == 1 and status(epi=5) == 1 and status(epi=7) == 1 and status(epi=2) == 1 and status(epi=3) == 1
    assert status(epi=2, r=P, ldr=8) == 2 and status(epi=2, r=P, ldr=16) == 0 and status(epi=2, r=ODD, ldr=16) == 1
    assert status(gate=C.c_void_p(4097)) == 1 and status(M=(1 << 20) + 1) == 2 and status(N=(1 << 24) + 8, ldc=1 << 25) == 2

    def status8(sa=P, **kw):
        v = list({**ok, **kw}.values())
        return lib.lvx_linear_fp8_fp4(v[0], v[1], sa, *v[2:], None)

    assert status8() == 0 and status8(sa=None) == 1 and status8(lda=72) == 2


def test_cache_sizes_and_refusals():
    lib = lvx.load()
    # per key and kv head: 64 bytes of codes for K and for V, 4 bytes of K's scales, 2 of V's; whole tiles of 64 keys
    assert lib.lvx_kv4_bytes(C.byref(lvx.kv4_desc(2, 3, 4, 128, 1000))) == 2 * 3 * 4 * 1024 * (64 + 64 + 4 + 2)
    assert lib.lvx_kv4_bytes(C.byref(lvx.kv4_desc(1, 1, 1, 64, 1))) == 64 * (32 + 32 + 2 + 2)
    for bad, st in ((dict(head_dim=96), 4), (dict(n_layers=0), 2), (dict(n_seqs=0), 2), (dict(n_kv_heads=0), 2), (dict(max_keys=0), 2),
                    (dict(n_seqs=65536), 2), (dict(max_keys=(1 << 26) + 1), 2)):
        d = dict(n_layers=2, n_seqs=3, n_kv_heads=4, head_dim=128, max_keys=1000)
        d.update(bad)
        desc, h = lvx.kv4_desc(**d), C.c_void_p()
        assert lib.lvx_kv4_bytes(C.byref(desc)) == 0
        assert lib.lvx_kv4_init(C.byref(desc), P, 1 << 60, C.byref(h)) == st
    huge = lvx.kv4_desc(2 ** 31 - 1, 65535, 1024, 128, 1 << 26)
    assert lib.lvx_kv4_bytes(C.byref(huge)) == 0 and b"2^62" in lib.lvx_last_error()
    desc, h = lvx.kv4_desc(2, 3, 4, 128, 1000), C.c_void_p()
    need = lib.lvx_kv4_bytes(C.byref(desc))
    assert lib.lvx_kv4_init(None, P, need, C.byref(h)) == 1 and lib.lvx_kv4_init(C.byref(desc), P, need, None) == 1
    assert lib.lvx_kv4_init(C.byref(desc), None, need, C.byref(h)) == 1 and lib.lvx_kv4_init(C.byref(desc), C.c_void_p(4096 + 16), need, C.byref(h)) == 1
    assert lib.lvx_kv4_init(C.byref(desc), P, need - 1, C.byref(h)) == 2
    assert lib.lvx_kv4_destroy(None) == 1


def test_cache_call_refusals():
    lib, h = lvx.load(), handle()
    ok = dict(c=h, layer=0, k=P, v=P, ld=512, starts=P, n=0, most=0, counts=P)

    def append(**kw):
        return lib.lvx_kv4_append(*{**ok, **kw}.values(), None)

    assert append() == 0 and append(starts=None) == 0
    assert append(c=None) == 1 and append(layer=2) == 1 and append(layer=-1) == 1 and append(k=None) == 1 and append(v=ODD) == 1
    assert append(counts=None) == 1 and append(counts=C.c_void_p(4097)) == 1 and append(starts=C.c_void_p(4098)) == 1
    assert append(ld=504) == 2 and append(ld=516) == 2 and append(n=-1) == 2 and append(most=-1) == 2
    assert append(n=4, most=1) == 2                          # more tokens than three sequences of one
    assert append(n=2, most=1, starts=None) == 2             # without starts all sequences have max_tokens
    ok_a = dict(c=h, layer=0, q=P, ldq=1024, heads=8, starts=P, n=0, most=0, counts=P, causal=1, scale=0.1, out=P, ldo=1024, ws=P, bytes=1 << 40)

    def attend(**kw):
        return lib.lvx_kv4_attention(*{**ok_a, **kw}.values(), None)

    assert attend() == 0
    assert attend(heads=6) == 2 and attend(heads=0) == 2 and attend(causal=2) == 1 and attend(q=ODD) == 1 and attend(out=None) == 1 and attend(ws=None) == 1
    assert attend(ldq=1016) == 2 and attend(ldo=1028) == 2 and attend(counts=None) == 1 and attend(n=10, most=3) == 2
    need = lib.lvx_kv4_attention_workspace_bytes(h, 8, 1)
    assert need >= 256
    assert lib.lvx_kv4_attention_workspace_bytes(h, 6, 1) == 0 and lib.lvx_kv4_attention_workspace_bytes(None, 8, 1) == 0
    assert lib.lvx_kv4_attention_workspace_bytes(h, 8, -1) == 0
    big = handle(max_keys=1 << 20)
    need = lib.lvx_kv4_attention_workspace_bytes(big, 8, 1)
    assert need > 256 and attend(c=big, n=3, most=1, bytes=need - 16) == 2
    g = lib.lvx_kv4_gather
    assert g(h, 0, 0, 0, P, P, P, 512, None) == 0
    assert g(h, 0, -1, 4, P, P, P, 512, None) == 2 and g(h, 0, 998, 3, P, P, P, 512, None) == 2 and g(h, 0, 0, 4, None, P, P, 512, None) == 1
    assert g(h, 0, 0, 4, P, ODD, P, 512, None) == 1 and g(h, 0, 0, 4, P, P, P, 504, None) == 2 and g(None, 0, 0, 4, P, P, P, 512, None) == 1
    for x in (h, big):
        assert lib.lvx_kv4_destroy(x) == 0


def test_workspace_never_shrinks_with_the_tokens():
    lib = lvx.load()
    for kw in (dict(), dict(max_keys=100000), dict(max_keys=100000, n_seqs=1, n_kv_heads=1), dict(max_keys=30000, n_seqs=1, n_kv_heads=8), dict(n_seqs=40, max_keys=5000)):
        h = handle(**kw)
        for heads in (1, 2, 5, 8):
            heads *= dict(n_kv_heads=4, **kw)["n_kv_heads"] if "n_kv_heads" not in kw else kw["n_kv_heads"]
            sizes = [lib.lvx_kv4_attention_workspace_bytes(h, heads, n) for n in range(0, 3000)]
            assert all(a <= b for a, b in zip(sizes, sizes[1:])), (kw, heads)
        lib.lvx_kv4_destroy(h)


def test_python_binding_refuses():
    with pytest.raises(lvx.LvxError):
        lvx.KV4Cache(lvx.kv4_desc(1, 1, 1, 96, 64), "cpu")


def test_python_binding_refuses_what_would_fault():
    """Tensors on the host, lengths of another type, too few of them or with gaps: refused before a launch."""
    import torch
    bf, i32 = torch.bfloat16, torch.int32
    w, s = torch.zeros(64, 32, dtype=torch.uint8), torch.zeros(64, 2, dtype=torch.uint8)
    x, c = torch.zeros(3, 64, dtype=bf), torch.zeros(3, 64, dtype=bf)
    for f in (lambda: lvx.lvx_linear_fp4(x, w, s, c), lambda: lvx.lvx_rmsnorm_residual(x, None, None, 1e-6, c), lambda: lvx.lvx_fp4_quantize(x)):
        with pytest.raises(lvx.LvxError, match="current device"):
            f()

    class Stub:
        desc, handle = lvx.kv4_desc(1, 3, 1, 64, 64), handle(n_layers=1, n_kv_heads=1, head_dim=64, max_keys=64)

    ws, good = torch.zeros(256, dtype=torch.uint8), torch.ones(3, dtype=i32)
    out = torch.zeros(3, 4, 64, dtype=bf)
    for counts, starts in ((torch.ones(3, dtype=torch.int64), None), (torch.ones(2, dtype=i32), None), (torch.ones(3, 2, dtype=i32)[:, 0], None),
                           (good, torch.zeros(3, dtype=i32)), (good, torch.zeros(4))):
        with pytest.raises(lvx.LvxError, match="int32"):
            lvx.lvx_kv4_append(Stub, 0, x, x, counts, starts=starts)
        with pytest.raises(lvx.LvxError, match="int32"):
            lvx.lvx_kv4_attention(Stub, 0, x, 1, 0.1, counts, c, ws, starts=starts)
        if starts is None:
            with pytest.raises(lvx.LvxError, match="int32"):
                lvx.lvx_kv4_gather(Stub, 0, counts, out, out.clone())
    with pytest.raises(lvx.LvxError, match="current device"):
        lvx.lvx_kv4_append(Stub, 0, x, x, good)
    with pytest.raises(lvx.LvxError, match="strides"):
        lvx.lvx_kv4_gather(Stub, 0, good, out, out[:, :2])
    lvx.lvx_kv4_gather(Stub, 0, good, out[:, :0], out[:, :0])
    lvx.lvx_rmsnorm_residual(x[:0], None, None, 1e-6, c[:0])


def test_mixed_products_are_for_8bit_rows_and_bf16_outputs():
    lib, flag = lvx.load(), lvx.EPI_MIXED_8X4
    a16 = (P, 64, P, 32, P, 2, P, 16, 0, 16, 64)
    a8 = (P, 64, P, P, 32, P, 2, P, 16, 0, 16, 64)
    for epi in (lvx.EPI_STORE, lvx.EPI_GELU_TANH, lvx.EPI_RESID_GATE):
        assert lib.lvx_linear_fp8_fp4(*a8, epi | flag, P, 16, None, None) == 0
        assert lib.lvx_linear_fp4(*a16, epi | flag, P, 16, None, None) == 1
    for epi in (lvx.EPI_RESID_GATE_F32, lvx.EPI_STORE_F32, lvx.EPI_BIAS, lvx.EPI_BIAS_SILU, 7, 16):
        assert lib.lvx_linear_fp8_fp4(*a8, epi | flag, P, 16, None, None) == (0 if epi == 16 else 1)
    assert lib.lvx_linear(P, 64, P, 64, P, 16, 8, 16, 64, flag, None, 0, None, None) == 1


@pytest.mark.parametrize("K,status", [(1 << 30, 0), ((1 << 30) + 32, 2), ((1 << 31) - 256, 2), ((1 << 31) - 32, 2)])
def test_more_channels_than_the_kernels_count(K, status):
    lib, ld = lvx.load(), 1 << 31
    assert lib.lvx_linear_fp4(P, ld, P, ld, P, ld, P, 16, 0, 16, K, 0, None, 0, None, None) == status
    assert lib.lvx_linear_fp8_fp4(P, ld, P, P, ld, P, ld, P, 16, 0, 16, K, 0, None, 0, None, None) == status
