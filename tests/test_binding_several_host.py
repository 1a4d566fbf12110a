"""The extension module's calls for several tokens per sequence on the host, with callbacks in the library's place: what is plain
reaches the library with the arguments of the ctypes calls, everything else is left to kvq.py."""
import ctypes as C
import importlib.util
import subprocess

import pytest
import torch

from paper_2502_15075_amd import build, kvq

P, I32, I64, F, SZ = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
SIGNATURES = {
    "rope_append": (P, P, P, I64, I64, I64, I32, P, P, P, C.c_int, I64, I64, I64, P, P, I32, C.POINTER(kvq._CRope), P),
    "chunk_attention": (P, P, P, C.c_int, I32, I64, I64, I64, I32, P, P, I32, I32, I32, F, P, C.c_int, P, SZ, P),
    "window_attention": (P, P, P, C.c_int, I32, P, I32, I32, I32, F, P, C.c_int, P, SZ, P),
}


@pytest.fixture(scope="module")
def bound(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("binding") / "_kvq_binding.so")
    r = subprocess.run(build.binding_command(so, "-DKVQ_CURRENT_STREAM()=nullptr"), capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    spec = importlib.util.spec_from_file_location("_kvq_binding", so)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    calls = []

    def entry(name):
        def call(*args):
            if name == "rope_append":                  # (the struct is the callee's only while it runs)
                r = args[17].contents
                args = args[:17] + ((r.cos, r.sin, r.rows, r.rotary_dim, r.interleaved),) + args[18:]
            calls.append((name, args))
            return 0
        return call
    functions = [C.CFUNCTYPE(C.c_int, *sig)(entry(name)) for name, sig in SIGNATURES.items()]
    module.bind(0, 0, 0, 0, 0, kvq.Layout, kvq.Cache)
    module.bind_several(*[C.cast(f, C.c_void_p).value for f in functions], kvq.Rope)
    module.ready()
    yield module, calls
    module.bind_several(0, 0, 0, kvq.Rope)


def plain_arguments():
    L = kvq.Layout(batch=2, kv_heads=2, max_seq=128, head_dim=128, bits_k=4, bits_v=2, group_k=64, group_v=64)
    cache = kvq.Cache(L, device="cpu", fill=0)
    h = lambda *s: torch.zeros(*s, dtype=torch.float16)
    lens = torch.ones(2, dtype=torch.int32)
    rope = kvq.Rope(torch.zeros(128, 64), torch.zeros(128, 64), True)
    return {
        "rope_append": [L, cache, h(2, 3, 6, 128)[:, :, 1:5], h(2, 2, 3, 128), h(2, 2, 3, 128), lens, rope, h(2, 3, 4, 128), lens.clone()],
        "chunk_attention": [L, cache, h(2, 4, 3, 128).transpose(1, 2), lens, lens.clone(), 100, 50, 3, 0.5, torch.zeros(2, 3, 4, 128), torch.zeros(64, dtype=torch.uint8)],
        "window_attention": [L, cache, h(2, 4, 128), lens, 100, 50, 3, 0.5, torch.zeros(2, 4, 128), torch.zeros(64, dtype=torch.uint8)],
    }


def test_arguments_arrive(bound):
    module, calls = bound
    a = plain_arguments()
    for name, args in a.items():
        calls.clear()
        assert getattr(module, name)(*args) == 0 and calls[0][0] == name
        got = calls[0][1]
        ptr = lambda i: args[i].data_ptr()
        if name == "rope_append":
            r = args[6]
            assert got[2:17] == (ptr(2), 3 * 6 * 128, 6 * 128, 128, 4, ptr(7), ptr(3), ptr(4), kvq.KVQ_F16, 768, 384, 128, ptr(5), ptr(8), 3)
            assert got[17] == (r.cos.data_ptr(), r.sin.data_ptr(), 128, 128, 1)
        elif name == "chunk_attention":
            assert got[2:19] == (ptr(2), kvq.KVQ_F16, 4, 1536, 128, 384, 3, ptr(3), ptr(4), 100, 50, 3, 0.5, ptr(9), kvq.KVQ_F32, ptr(10), 64)
        else:
            assert got[2:14] == (ptr(2), kvq.KVQ_F16, 4, ptr(3), 100, 50, 3, 0.5, ptr(8), kvq.KVQ_F32, ptr(9), 64)


def test_what_may_be_none(bound):
    module, calls = bound
    a = plain_arguments()
    for name, nones in (("rope_append", (2, 7)), ("rope_append", (8,)), ("chunk_attention", (3, 4, 10)), ("window_attention", (3, 9))):
        args = list(a[name])
        for i in nones:
            args[i] = None
        calls.clear()
        assert getattr(module, name)(*args) == 0 and len(calls) == 1


@pytest.mark.parametrize("name", SIGNATURES)
def test_what_is_not_plain_is_left(bound, name):
    """Each argument in turn of another kind, form, type or shape."""
    module, calls = bound
    for i, arg in enumerate(plain_arguments()[name]):
        worse = [object(), "x"]
        if isinstance(arg, torch.Tensor):
            worse += [arg.double(), arg[:1]] + ([arg.unsqueeze(0)] if arg.dim() > 1 else [])
            if arg.dim() > 1:
                worse += [torch.zeros(*arg.shape[:-1], 256, dtype=arg.dtype)[..., ::2], arg.numpy()]
            if arg.dtype == torch.uint8:
                worse = [object(), "x"]
        elif isinstance(arg, int):
            worse += [1 << 40, 1.5, None]
        elif isinstance(arg, float):
            worse += [1, None]
        for bad in worse:
            args = list(plain_arguments()[name])
            args[i] = bad
            calls.clear()
            assert getattr(module, name)(*args) is None and not calls, (i, bad)
    args = plain_arguments()[name]
    assert getattr(module, name)(*args[:-1]) is None and getattr(module, name)(*args, None) is None
