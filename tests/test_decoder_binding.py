"""Every tensor that the decoder operators' binding hands to the library has to lie on the current device, with the type and the extents that the kernels
take: one argument is misplaced at a time, the library is a stub that counts its calls, and no GPU is needed."""
import pytest
import torch

import paper_2512_04677_amd as lvx

BF, F32, U8, I32 = torch.bfloat16, torch.float32, torch.uint8, torch.int32


class On:
    """A host tensor that says it lies on a device."""

    def __init__(self, t, device=0):
        self.t, self.on = t, device

    def get_device(self):
        return self.on

    @property
    def device(self):
        return "device %d" % self.on

    def __getattr__(self, name):
        return getattr(self.t, name)


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


@pytest.fixture
def stub(monkeypatch):
    lib = Library()
    monkeypatch.setattr(lvx, "load", lambda: lib)
    monkeypatch.setattr(lvx, "_here", lambda: (0, 77))
    return lib


def rows(n, d, dtype=BF, pad=8):
    return torch.zeros(n, d + pad, dtype=dtype)[:, :d]


class Cache:
    desc, handle = lvx.kv4_desc(1, 3, 2, 64, 100), 5

    def __init__(self):
        self.storage = On(torch.zeros(1, dtype=U8))


M, N, K = 3, 24, 64


def calls():
    """name -> (function of the tensors, the tensors by name); matrices are named (name, rows, columns)."""
    w = dict(wq=torch.zeros(N, K // 2, dtype=U8), w_scales=rows(N, K // 32, U8))
    flat = torch.zeros
    out = {}
    for kind, f32 in (("bf16", False), ("f32", True)):
        r = F32 if f32 else BF
        epi = lvx.EPI_RESID_GATE_F32 if f32 else lvx.EPI_RESID_GATE
        norm = dict(x=rows(M, K), resid=rows(M, K, r), gain=flat(K), sum_out=rows(M, K, r))
        out["norm " + kind] = (lambda **t: lvx.lvx_rmsnorm_residual(t["x"], t["resid"], t["gain"], 1e-6, t["y"], sum_out=t["sum_out"]), dict(norm, y=rows(M, K)))
        out["norm8 " + kind] = (lambda **t: lvx.lvx_rmsnorm_residual_fp8(t["x"], t["resid"], t["gain"], 1e-6, t["y"], t["row_scales"], sum_out=t["sum_out"]),
                                dict(norm, y=rows(M, K, U8, 16), row_scales=flat(M)))
        tail = dict(c=rows(M, N, r), resid=rows(M, N, r), gate=flat(N))
        out["linear " + kind] = (lambda epi=epi, **t: lvx.lvx_linear_fp4(t["a"], t["wq"], t["w_scales"], t["c"], epi, resid=t["resid"], gate=t["gate"]),
                                 dict(w, a=rows(M, K), **tail))
        out["linear8 " + kind] = (lambda epi=epi, **t: lvx.lvx_linear_fp8_fp4(t["a"], t["row_scales"], t["wq"], t["w_scales"], t["c"], epi, resid=t["resid"], gate=t["gate"]),
                                  dict(w, a=rows(M, K, U8, 16), row_scales=flat(M), **tail))
    out["quantize"] = (lambda **t: lvx.lvx_fp4_quantize(t["x"], t["q"], t["scales"]), dict(x=rows(M, K), q=rows(M, K // 2, U8, 16), scales=rows(M, K // 32, U8)))
    counts = dict(counts=torch.ones(3, dtype=I32), starts=torch.zeros(4, dtype=I32))
    out["append"] = (lambda cache=None, **t: lvx.lvx_kv4_append(cache or Cache(), 0, t["k"], t["v"], t["counts"], starts=t["starts"], n_tokens=M), dict(counts, k=rows(M, 128), v=rows(M, 128)))
    out["gather"] = (lambda cache=None, **t: lvx.lvx_kv4_gather(cache or Cache(), 0, t["counts"], t["k_out"], t["v_out"]),
                     dict(counts=counts["counts"], k_out=flat(3, 5, 136, dtype=BF)[:, :, :128], v_out=flat(3, 5, 136, dtype=BF)[:, :, :128]))
    out["attention"] = (lambda cache=None, **t: lvx.lvx_kv4_attention(cache or Cache(), 0, t["q"], 4, 0.1, t["counts"], t["out"], t["workspace"], starts=t["starts"], n_tokens=M),
                        dict(counts, q=rows(M, 256), out=rows(M, 256), workspace=flat(256, dtype=U8)))
    return out


def every():
    return [(name, arg) for name, (_, tensors) in calls().items() for arg in tensors]


def test_good_calls_reach_the_library(stub):
    for name, (f, tensors) in calls().items():
        stub.calls.clear()
        f(**{k: On(t) for k, t in tensors.items()})
        assert len(stub.calls) == 1, name
        args = stub.calls[0][1]
        assert args[-1] == 77 and all(t.data_ptr() in args for t in tensors.values()), name


@pytest.mark.parametrize("name,arg", every())
@pytest.mark.parametrize("where", [-1, 1])
def test_one_tensor_elsewhere(stub, name, arg, where):
    f, tensors = calls()[name]
    with pytest.raises(lvx.LvxError, match="device"):
        f(**{k: On(t, where if k == arg else 0) for k, t in tensors.items()})
    assert not stub.calls


@pytest.mark.parametrize("name", ["append", "gather", "attention"])
def test_the_cache_elsewhere(stub, name):
    f, tensors = calls()[name]
    cache = Cache()
    cache.storage.on = 1
    with pytest.raises(lvx.LvxError, match="device"):
        f(cache=cache, **{k: On(t) for k, t in tensors.items()})
    assert not stub.calls


@pytest.mark.parametrize("name,arg", [(n, a) for n, a in every() if a != "workspace"])
def test_one_tensor_of_another_type(stub, name, arg):
    f, tensors = calls()[name]
    for dtype in (torch.float16, torch.int32 if tensors[arg].dtype != I32 else torch.int64, F32 if tensors[arg].dtype == BF else BF):
        if name.startswith("norm") and arg == "resid" and dtype in (F32, BF):
            continue  # the residual's type is its own choice; the sum then has to follow
        with pytest.raises(lvx.LvxError):
            f(**{k: On(t.to(dtype) if k == arg else t) for k, t in tensors.items()})
    assert not stub.calls


def shrunk(t):
    """The tensor with a row or element too few, with a column too few, and with gaps between its columns."""
    if t.dim() == 1:
        return [t[:-1], torch.zeros(2 * len(t), dtype=t.dtype)[::2]]
    wide = torch.zeros(*t.shape[:-1], 2 * t.shape[-1], dtype=t.dtype)
    return [t[:-1], t[..., :-1], wide[..., ::2]]


@pytest.mark.parametrize("name,arg", every())
def test_one_tensor_too_small_or_with_gaps(stub, name, arg):
    f, tensors = calls()[name]
    for i, bad in enumerate(shrunk(tensors[arg])):
        if arg == "workspace" and i == 0:
            continue  # its bytes are passed on: the library compares them
        if name.split()[0] in ("linear", "linear8", "norm", "norm8", "quantize") and arg in ("a", "x") and i == 0:
            continue  # fewer rows: a smaller call (the norm's residual then differs)
        if name == "quantize" and arg == "x" and i == 1:
            continue  # x says the sizes; 63 columns are the library's to refuse
        with pytest.raises(lvx.LvxError):
            f(**{k: On(bad if k == arg else t) for k, t in tensors.items()})
    assert not stub.calls


def test_weights_of_another_width(stub):
    f, tensors = calls()["linear bf16"]
    t = {k: On(v) for k, v in tensors.items()}
    for kw in (dict(a=On(rows(M, 2 * K))), dict(wq=On(torch.zeros(N, K, dtype=U8))), dict(w_scales=On(rows(N, 4, U8))), dict(w_scales=On(rows(N + 8, 2, U8)))):
        with pytest.raises(lvx.LvxError):
            f(**{**t, **kw})
    with pytest.raises(lvx.LvxError):
        lvx.lvx_linear_fp4(t["a"], t["wq"], t["w_scales"], t["c"], lvx.EPI_RESID_GATE_F32, resid=t["resid"])   # bf16 residual and output for the fp32 epilogue
    with pytest.raises(lvx.LvxError):
        lvx.lvx_rmsnorm_residual(None, None, None, 1e-6, On(rows(M, K)))
    assert not stub.calls
    lvx.lvx_linear_fp8_fp4(On(rows(M, K, U8, 16).view(torch.float8_e4m3fn)), On(torch.zeros(M)), t["wq"], t["w_scales"], t["c"])
    assert len(stub.calls) == 1


def test_more_tokens_than_rows(stub):
    t = {k: On(v) for k, v in calls()["append"][1].items()}
    with pytest.raises(lvx.LvxError):
        lvx.lvx_kv4_append(Cache(), 0, t["k"], t["v"], t["counts"], starts=t["starts"], n_tokens=M + 1)
    t = {k: On(v) for k, v in calls()["attention"][1].items()}
    with pytest.raises(lvx.LvxError):
        lvx.lvx_kv4_attention(Cache(), 0, t["q"], 4, 0.1, t["counts"], t["out"], t["workspace"], starts=t["starts"], n_tokens=M + 1)
    with pytest.raises(lvx.LvxError):
        lvx.lvx_kv4_attention(Cache(), 0, t["q"], 6, 0.1, t["counts"], t["out"], t["workspace"], starts=t["starts"], n_tokens=M)
    assert not stub.calls


def test_heads_as_a_dimension(stub):
    """[tokens][heads][channels] is the same memory as [tokens][heads * channels] where it has no gaps inside a token."""
    c = calls()["append"][1]
    k, v = torch.zeros(M, 2, 64, dtype=BF), torch.zeros(M, 2, 64, dtype=BF)
    counts, starts = On(c["counts"]), On(c["starts"])
    lvx.lvx_kv4_append(Cache(), 0, On3(k), On3(v), counts, starts=starts)
    q, out = torch.zeros(M, 6, 64, dtype=BF)[:, :4], torch.zeros(M, 4, 64, dtype=BF)
    lvx.lvx_kv4_attention(Cache(), 0, On3(q), 4, 0.1, counts, On3(out), On(torch.zeros(256, dtype=U8)), starts=starts)
    assert [a[2:5] for _, a in stub.calls] == [(k.data_ptr(), v.data_ptr(), 128), (q.data_ptr(), 384, 4)]
    stub.calls.clear()
    for bad in (torch.zeros(M, 2, 72, dtype=BF)[:, :, :64], torch.zeros(M, 64, 2, dtype=BF).transpose(1, 2), torch.zeros(2, M, 64, dtype=BF).transpose(0, 1), k[0]):
        with pytest.raises(lvx.LvxError):
            lvx.lvx_kv4_append(Cache(), 0, On3(k), On3(bad), counts, starts=starts, n_tokens=M)
    assert not stub.calls


class On3(On):
    def flatten(self, first):
        return On(self.t.flatten(first))


def test_bytes_by_their_torch_types(stub):
    w, s = torch.zeros(N, K // 2, dtype=U8), torch.zeros(N, K // 32, dtype=U8)
    for name, t in (("float4_e2m1fn_x2", "w"), ("float8_e8m0fnu", "s")):
        dtype = getattr(torch, name, None)
        if dtype is None:
            continue
        f = lambda x, which: On(x.view(dtype)) if t == which else On(x)
        lvx.lvx_linear_fp4(On(rows(M, K)), f(w, "w"), f(s, "s"), On(rows(M, N)))
        lvx.lvx_fp4_quantize(On(rows(N, K)), f(w, "w"), f(s, "s"))
    lvx.lvx_rmsnorm_residual_fp8(On(rows(M, K)), None, None, 1e-6, On(torch.zeros(M, K, dtype=U8).view(torch.float8_e4m3fn)), On(torch.zeros(M)))
    assert len(stub.calls) == 1 + 2 * sum(hasattr(torch, n) for n in ("float4_e2m1fn_x2", "float8_e8m0fnu"))
