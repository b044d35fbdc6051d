"""The layer's entry points without a GPU: refusals before anything is launched,
and the native marshalling of their arguments."""
import ctypes
import inspect
import os
import re
import subprocess

import pytest

torch = pytest.importorskip("torch")

from paper_2607_26444_amd import build, moe  # noqa: E402

A = ctypes.c_void_p(0x10000)      # never followed: the calls are refused
MIS = ctypes.c_void_p(0x10004)
WS = ctypes.c_void_p(0x100000)
NAN, INF = float("nan"), float("inf")


def _refuses(fn, good, cases):
    for change, code in cases:
        bad = dict(good, **change)
        assert getattr(moe.lib(), fn)(*bad.values()) == code, (fn, change)


ROUTE = dict(x=A, dtype=2, pitch=0, T=8, k=4, E=64, score=0, bias=None, groups=1, top=1, two=1,
             renorm=1, scale=1.0, mask=None, idx=A, w=A, stream=None)


def test_route_refusals():
    E, L = moe.MOE_EINVAL, moe.MOE_EALIGN
    _refuses("moe_route", ROUTE, [
        (dict(x=None), E), (dict(idx=None), E), (dict(w=None), E), (dict(T=-1), E), (dict(k=0), E),
        (dict(k=33), E), (dict(k=65, E=64), E), (dict(E=0), E), (dict(E=1025), E), (dict(dtype=1), E),
        (dict(dtype=3), E), (dict(pitch=63), E), (dict(pitch=-1), E), (dict(score=2), E),
        (dict(scale=NAN), E), (dict(scale=INF), E), (dict(groups=0), E), (dict(groups=65, E=65), E),
        (dict(groups=5), E), (dict(groups=8, top=9), E), (dict(groups=8, top=0), E),
        (dict(two=0), E), (dict(two=3), E), (dict(groups=32, top=1), E), (dict(T=2 ** 30), E),
        (dict(x=ctypes.c_void_p(0x10002)), L), (dict(idx=ctypes.c_void_p(0x10002)), L),
        (dict(bias=ctypes.c_void_p(0x10002)), L)])
    assert moe.lib().moe_route(*dict(ROUTE, T=0, x=None, idx=None, w=None).values()) == moe.MOE_OK


def test_route_backward_refusals():
    E = moe.MOE_EINVAL
    good = dict(x=A, dtype=2, pitch=0, T=8, k=4, E=64, score=0, renorm=1, scale=1.0, idx=A, g=A,
                out=A, stream=None)
    _refuses("moe_route_backward", good, [
        (dict(x=None), E), (dict(idx=None), E), (dict(g=None), E), (dict(out=None), E), (dict(k=0), E),
        (dict(dtype=1), E), (dict(score=-1), E), (dict(pitch=10), E), (dict(scale=NAN), E),
        (dict(out=ctypes.c_void_p(0x10002)), moe.MOE_EALIGN)])
    assert moe.lib().moe_route_backward(*dict(good, T=0, x=None).values()) == moe.MOE_OK


def test_rmsnorm_refusals():
    E, L = moe.MOE_EINVAL, moe.MOE_EALIGN
    good = dict(x=A, xp=0, r=A, rd=0, rp=0, w=A, wd=0, eps=1e-6, T=8, H=1024, s=A, y=A, qd=1, q=A,
                qs=A, cols=0, rstd=A, stream=None)
    _refuses("moe_rmsnorm", good, [
        (dict(x=None), E), (dict(w=None), E), (dict(T=-1), E), (dict(H=0), E), (dict(H=16392), E),
        (dict(eps=-1.0), E), (dict(eps=NAN), E), (dict(wd=1), E), (dict(rd=3), E), (dict(r=None), E),
        (dict(s=None, y=None, q=None, rstd=None), E), (dict(qs=None), E), (dict(qd=0), E),
        (dict(qd=2), E), (dict(cols=9), E), (dict(cols=-1), E), (dict(xp=1016), E), (dict(rp=8), E),
        (dict(s=A, rp=1032), E),                       # in place wants packed rows
        (dict(H=1020, q=None), L), (dict(H=1032), L), (dict(H=1032, qd=3), L), (dict(xp=1028), L),
        (dict(rp=1028, s=None), L), (dict(x=MIS), L), (dict(r=MIS), L), (dict(w=MIS), L), (dict(y=MIS), L),
        (dict(q=MIS), L), (dict(s=MIS), L), (dict(rstd=ctypes.c_void_p(0x10001)), L)])
    assert moe.lib().moe_rmsnorm(*dict(good, T=0, x=None).values()) == moe.MOE_OK


def test_quantize_refusals():
    E, L = moe.MOE_EINVAL, moe.MOE_EALIGN
    good = dict(x=A, xp=0, rows=8, H=1024, src=None, qd=3, q=A, qs=A, cols=0, stream=None)
    _refuses("moe_quantize", good, [
        (dict(x=None), E), (dict(q=None), E), (dict(qs=None), E), (dict(rows=-1), E), (dict(H=0), E),
        (dict(H=16400), E), (dict(qd=0), E), (dict(xp=8), E), (dict(cols=-2), E), (dict(H=1032), L),
        (dict(H=1040, qd=1), L), (dict(x=MIS), L), (dict(q=MIS), L),
        (dict(src=ctypes.c_void_p(0x10001)), L)])
    assert moe.lib().moe_quantize(*dict(good, rows=0, x=None).values()) == moe.MOE_OK


def test_rmsnorm_backward_refusals():
    E, L = moe.MOE_EINVAL, moe.MOE_EALIGN
    n = moe.moe_rmsnorm_backward_workspace_bytes(100, 1024)
    assert n >= 1024 * 4
    good = dict(gy=A, h=A, hd=0, rstd=A, w=A, wd=0, gs=None, T=100, H=1024, gx=A, gw=A, ws=WS, n=n,
                stream=None)
    _refuses("moe_rmsnorm_backward", good, [
        (dict(gy=None), E), (dict(h=None), E), (dict(rstd=None), E), (dict(w=None), E),
        (dict(gx=None), E), (dict(hd=1), E), (dict(wd=3), E), (dict(H=0), E), (dict(T=-1), E),
        (dict(H=16392), E), (dict(H=1020), L), (dict(gy=MIS), L), (dict(h=MIS), L), (dict(gx=MIS), L),
        (dict(gs=MIS), L), (dict(ws=None), moe.MOE_EWORKSPACE), (dict(n=n - 1), moe.MOE_EWORKSPACE),
        (dict(ws=ctypes.c_void_p(0x100010)), moe.MOE_EWORKSPACE)])
    out = ctypes.c_size_t()
    assert moe.lib().moe_rmsnorm_backward_workspace_bytes(8, 1024, None) == E
    assert moe.lib().moe_rmsnorm_backward_workspace_bytes(8, 12, ctypes.byref(out)) == L
    assert moe.lib().moe_rmsnorm_backward(*dict(good, T=0, gw=None, ws=None, n=0).values()) == 0


def test_expert_matmul_refusals():
    E, L = moe.MOE_EINVAL, moe.MOE_EALIGN
    good = dict(a=A, sa=A, sp=0, rows=8, w=A, sw=A, E=4, N=64, K=128, off=A, cnt=A, act=0, y=A,
                stream=None)
    _refuses("moe_expert_matmul", good, [
        (dict(a=None), E), (dict(sa=None), E), (dict(w=None), E), (dict(sw=None), E), (dict(y=None), E),
        (dict(rows=-1), E), (dict(rows=2 ** 31), E), (dict(E=0), E), (dict(E=1025), E), (dict(N=0), E),
        (dict(K=0), E), (dict(K=131072), E), (dict(act=2), E), (dict(off=None), E),
        (dict(off=None, E=1), E),                      # counts without offsets
        (dict(sp=-1), E), (dict(K=120), L), (dict(N=60), L), (dict(N=72, act=1), L), (dict(a=MIS), L),
        (dict(w=MIS), L), (dict(y=MIS), L), (dict(off=ctypes.c_void_p(0x10001)), L)])
    assert moe.lib().moe_expert_matmul(*dict(good, rows=0, a=None).values()) == moe.MOE_OK


# ------------------------------------------------------------- marshalling
NAMES = ("moe_route", "moe_route_backward", "moe_rmsnorm", "moe_rmsnorm_backward", "moe_quantize",
         "moe_expert_matmul")
OTHERS = ("moe_layout", "moe_layout_fixed", "moe_dispatch", "moe_combine", "moe_layout_dedup",
          "moe_dispatch_dedup", "moe_expand", "moe_combine_local", "moe_combine_dedup")


def _prototypes():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(build.INCLUDE, "moe.h")).read(), flags=re.S)
    out = {}
    for name in NAMES + OTHERS:
        args = re.search(rf"\bint {name}\(([^)]*)\);", text).group(1)
        out[name] = [re.match(r"(.*?)(\w+)$", " ".join(a.split())).groups()
                     for a in args.split(",")]
    return out


PROTO = _prototypes()


class Buf:
    is_cuda = True

    def __init__(self, addr, shape=None):
        self.addr, self.shape = addr, shape

    def data_ptr(self):
        return self.addr

    def numel(self):
        return self.addr // 16 + 3

    def element_size(self):
        return 4


class Stream:
    cuda_stream = 0x7F00DEADB000


T, K = (1 << 33) + 5, 31
LONG = {"rows", "x_pitch", "residual_pitch", "logits_pitch", "T"}


def _arguments(name):
    """A value of its own for every parameter of a wrapper."""
    kinds = {p: t for t, p in PROTO[name]}
    args = {}
    for i, p in enumerate(inspect.signature(getattr(moe, name)).parameters):
        if p == "stream":
            args[p] = Stream()
        elif p == "workspace" or "*" in kinds[p]:
            args[p] = Buf(0x7F0000000000 + 0x1000 * (i + 1), (T, K) if p == "topk_idx" else None)
        elif kinds[p].startswith("float"):
            args[p] = 1.0 + i / 64
        else:
            args[p] = ((1 << 33) if p in LONG else 100) + i
    return args


def _expected(name, args):
    out = []
    for ctype, p in PROTO[name]:
        if p == "T" and "T" not in args:
            out.append(T)
        elif p == "k":
            out.append(K)
        elif p == "workspace_bytes":
            out.append(args["workspace"].numel() * 4 if args["workspace"] else 0)
        elif p == "stream":
            out.append(args[p].cuda_stream)
        else:
            v = args[p]
            out.append(0 if v is None else v.addr if isinstance(v, Buf) else v)
    return out


@pytest.fixture(scope="module")
def stub(tmp_path_factory):
    d = tmp_path_factory.mktemp("stub")
    src, so = os.path.join(d, "stub.cpp"), os.path.join(d, "libstub_layer.so")
    with open(src, "w") as f:
        f.write('#include "moe.h"\nextern "C" { double num[32]; unsigned long long rec[32]; '
                'int n_rec, code; }\n')
        for name, params in PROTO.items():
            f.write(f'extern "C" int {name}({", ".join(t + p for t, p in params)}) {{\n  n_rec = 0;\n')
            for t, p in params:
                if t.startswith("float ") and "*" not in t:
                    f.write(f"  num[n_rec] = {p}; rec[n_rec++] = 0;\n")
                else:
                    f.write(f"  num[n_rec] = -1; rec[n_rec++] = (unsigned long long){p};\n")
            f.write("  return code;\n}\n")
    subprocess.run(["g++", "-shared", "-fPIC", "-I", build.INCLUDE, src, "-o", so], check=True)
    lib = ctypes.CDLL(so)
    calls = moe._calls()
    calls.init(so, ctypes.ArgumentError, ctypes.c_int, lambda: 3,
               lambda dev: Stream.cuda_stream + 0x40)

    class Stub:
        code = ctypes.c_int.in_dll(lib, "code")

        @staticmethod
        def recorded():
            n = ctypes.c_int.in_dll(lib, "n_rec").value
            ints = list((ctypes.c_ulonglong * 32).in_dll(lib, "rec"))[:n]
            nums = list((ctypes.c_double * 32).in_dll(lib, "num"))[:n]
            return [i if x == -1 else x for i, x in zip(ints, nums)]

    yield Stub
    calls.init(moe.LIB_PATH, ctypes.ArgumentError, ctypes.c_int, torch._C._cuda_getDevice,
               torch._C._cuda_getCurrentRawStream)


@pytest.mark.parametrize("name", NAMES)
def test_every_argument_arrives(stub, name):
    args = _arguments(name)
    getattr(moe, name)(**args)
    assert stub.recorded() == _expected(name, args)


@pytest.mark.parametrize("name", NAMES)
def test_none_is_null(stub, name):
    for p, v in _arguments(name).items():
        if isinstance(v, Buf) and p != "topk_idx":
            args = dict(_arguments(name), **{p: None})
            getattr(moe, name)(**args)
            assert stub.recorded() == _expected(name, args), p


@pytest.mark.parametrize("name", NAMES)
def test_current_stream_and_error(stub, name):
    args = _arguments(name)
    del args["stream"]
    getattr(moe, name)(**args)
    assert stub.recorded()[-1] == Stream.cuda_stream + 0x40
    stub.code.value = moe.MOE_EALIGN
    try:
        with pytest.raises(moe.MoeError, match=name):
            getattr(moe, name)(**args)
    finally:
        stub.code.value = 0


def test_wrong_numbers(stub):
    with pytest.raises(TypeError):
        moe.moe_route(**dict(_arguments("moe_route"), scale="x"))
    with pytest.raises(ctypes.ArgumentError):
        moe.moe_quantize(**dict(_arguments("moe_quantize"), rows=1.5))
    with pytest.raises(TypeError):
        moe._calls().route(1, 2)


def test_a_library_without_the_layer_says_so(stub, tmp_path):
    src, so = tmp_path / "old.cpp", tmp_path / "libold.so"
    src.write_text('#include "moe.h"\n' + "".join(
        f'extern "C" int {n}({", ".join(t + p for t, p in PROTO[n])}) {{ return 0; }}\n'
        for n in OTHERS))
    subprocess.run(["g++", "-shared", "-fPIC", "-w", "-I", build.INCLUDE, str(src), "-o", str(so)],
                   check=True)
    lib = ctypes.CDLL(str(so))
    calls = moe._calls()
    calls.init(str(so), ctypes.ArgumentError, ctypes.c_int, lambda: 0, lambda dev: 0)
    with pytest.raises(RuntimeError, match="moe_route"):
        moe.moe_route(**_arguments("moe_route"))
    assert lib


def test_calls_of_no_rows_take_empty_tensors():
    """An empty tensor's address is null, whatever a program holds beside it: no call of
    no rows may ask for it, and none starts anything."""
    ok, L = moe.MOE_OK, moe.lib()
    assert L.moe_quantize(None, 0, 0, 1024, None, 3, None, None, 0, None) == ok
    assert L.moe_quantize(None, 0, 0, 1024, None, 3, A, None, 0, None) == ok
    assert L.moe_quantize(None, 0, 0, 1024, None, 1, None, A, 0, None) == ok
    good = dict(x=None, xp=0, r=A, rd=0, rp=0, w=A, wd=0, eps=1e-6, T=0, H=1024, s=A, y=A, qd=1, q=A,
                qs=A, cols=0, rstd=A, stream=None)
    for change in (dict(r=None), dict(qs=None), dict(q=None), dict(s=None, y=None, q=None, rstd=None)):
        assert L.moe_rmsnorm(*dict(good, **change).values()) == ok, change
    # what has nothing to do with the rows is still looked at
    E, M = moe.MOE_EINVAL, moe.MOE_EALIGN
    assert L.moe_quantize(None, 0, 0, 1024, None, 0, None, None, 0, None) == E
    assert L.moe_quantize(None, 0, 0, 1032, None, 3, None, None, 0, None) == M
    assert L.moe_quantize(None, 0, 0, 1040, None, 1, None, None, 0, None) == M
    assert L.moe_quantize(None, 0, 0, 1024, None, 3, MIS, None, 0, None) == M
    assert L.moe_quantize(None, 0, 0, 1024, None, 1, None, None, 9, None) == E
    for change, code in ((dict(w=None), E), (dict(H=16392), E), (dict(eps=NAN), E), (dict(H=1032), M),
                         (dict(qd=2), E), (dict(cols=9), E)):
        assert L.moe_rmsnorm(*dict(good, **change).values()) == code, change


def test_dispatch_of_no_tokens_takes_empty_scales():
    good = dict(x=None, xs=None, dtype=1, T=0, H=1024, k=2, E=8, R=1, idx=None, pos=None, ro=A, rx=A,
                rs=A, pitch=0, cap=A, ws=WS, n=1 << 30, status=A, stream=None)
    assert moe.lib().moe_dispatch(*good.values()) == moe.MOE_OK
    _refuses("moe_dispatch", good, [(dict(T=8, x=A, idx=A, pos=A), moe.MOE_EINVAL),
                                    (dict(rs=None), moe.MOE_EINVAL)])
