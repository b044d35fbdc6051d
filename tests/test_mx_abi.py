"""The balance loss's and the 4-bit floats' entry points without a GPU: refusals before
anything is launched, and the native marshalling of their arguments."""
import ctypes
import inspect
import os
import re
import subprocess

import pytest

torch = pytest.importorskip("torch")

import test_layer_abi as base  # noqa: E402
from paper_2607_26444_amd import build, moe  # noqa: E402

A, WS, Buf, Stream = base.A, base.WS, base.Buf, base.Stream
ODD = ctypes.c_void_p(0x10001)
TWO = ctypes.c_void_p(0x10002)
MIS = base.MIS
E, L, W = moe.MOE_EINVAL, moe.MOE_EALIGN, moe.MOE_EWORKSPACE

BALANCE = dict(x=A, dtype=2, pitch=0, T=4096, k=4, E=64, score=0, seq=0, idx=A, mask=None, count=A,
               live=A, mean=A, loss=A, ws=WS, n=1 << 30, stream=None)


def test_balance_refusals():
    base._refuses("moe_balance", BALANCE, [
        (dict(x=None), E), (dict(idx=None), E), (dict(count=None), E), (dict(live=None), E),
        (dict(T=-1), E), (dict(k=0), E), (dict(k=33), E), (dict(k=5, E=4), E), (dict(E=0), E),
        (dict(E=1025), E), (dict(dtype=1), E), (dict(dtype=3), E), (dict(pitch=63), E),
        (dict(pitch=-1), E), (dict(score=2), E), (dict(seq=-1), E), (dict(seq=4097), E),
        (dict(seq=1000), E), (dict(T=2 ** 30), E), (dict(x=TWO), L), (dict(dtype=0, x=ODD), L),
        (dict(idx=TWO), L), (dict(count=TWO), L), (dict(live=TWO), L), (dict(mean=TWO), L),
        (dict(loss=TWO), L), (dict(ws=None), W), (dict(ws=MIS), W), (dict(n=100), W)])
    assert moe.lib().moe_balance(*dict(BALANCE, T=0, seq=8, x=None, idx=None).values()) == moe.MOE_OK


def test_balance_workspace():
    out = ctypes.c_size_t(0)
    ask = moe.lib().moe_balance_workspace_bytes
    for T, n, seq in ((-1, 64, 0), (8, 0, 0), (8, 1025, 0), (8, 64, -1), (8, 64, 3), (2 ** 31, 64, 0)):
        assert ask(T, n, seq, ctypes.byref(out)) == E
    assert ask(8, 64, 0, None) == E
    assert moe.moe_balance_workspace_bytes(8, 64) == 0           # one part
    assert moe.moe_balance_workspace_bytes(0, 64) == 0
    need = moe.moe_balance_workspace_bytes(32768, 256)
    assert 0 < need < 8 << 20
    base._refuses("moe_balance", dict(BALANCE, T=32768, E=256, n=need - 1), [({}, W)])


def test_balance_backward_refusals():
    good = dict(x=A, dtype=2, pitch=0, T=64, E=64, score=0, seq=0, mask=None, count=A, live=A, gl=A,
                gs=None, out=A, stream=None)
    base._refuses("moe_balance_backward", good, [
        (dict(x=None), E), (dict(count=None), E), (dict(live=None), E), (dict(gl=None), E),
        (dict(out=None), E), (dict(T=-1), E), (dict(E=0), E), (dict(E=1025), E), (dict(dtype=1), E),
        (dict(pitch=63), E), (dict(score=-1), E), (dict(seq=-1), E), (dict(seq=63), E),
        (dict(x=TWO), L), (dict(gs=TWO), L), (dict(out=TWO), L), (dict(dtype=0, out=ODD), L),
        (dict(count=TWO), L), (dict(live=TWO), L), (dict(gl=TWO), L)])
    none = dict.fromkeys(("x", "count", "live", "gl", "out"))
    assert moe.lib().moe_balance_backward(*dict(good, T=0, **none).values()) == moe.MOE_OK


def test_quantize_mx_refusals():
    good = dict(x=A, xp=0, rows=8, H=256, src=None, q=A, qp=0, s=A, sp=0, v=A, stream=None)
    base._refuses("moe_quantize_mx", good, [
        (dict(x=None), E), (dict(q=None), E), (dict(s=None), E), (dict(rows=-1), E),
        (dict(rows=2 ** 31), E), (dict(H=0), E), (dict(H=131072), E), (dict(xp=248), E),
        (dict(xp=-8), E), (dict(xp=2 ** 31), E), (dict(qp=112), E), (dict(qp=-16), E),
        (dict(sp=4), E), (dict(sp=-4), E), (dict(qp=2 ** 31), E), (dict(sp=2 ** 31), E),
        (dict(H=264), L), (dict(H=16), L), (dict(xp=260), L), (dict(qp=136), L), (dict(sp=10), L),
        (dict(x=MIS), L), (dict(q=MIS), L), (dict(s=TWO), L), (dict(v=MIS), L), (dict(src=TWO), L)])
    none = dict.fromkeys(("x", "q", "s", "v"))
    assert moe.lib().moe_quantize_mx(*dict(good, rows=0, **none).values()) == moe.MOE_OK


def test_expert_matmul_mx_refusals():
    good = dict(a=A, ap=0, sa=A, sp=0, rows=8, w=A, sw=A, E=4, N=64, K=288, off=A, cnt=A, act=0, y=A,
                stream=None)
    base._refuses("moe_expert_matmul_mx", good, [
        (dict(a=None), E), (dict(sa=None), E), (dict(w=None), E), (dict(sw=None), E), (dict(y=None), E),
        (dict(rows=-1), E), (dict(rows=2 ** 31), E), (dict(E=0), E), (dict(E=1025), E), (dict(N=0), E),
        (dict(N=moe.MOE_MAX_MX_CHANNELS + 16), E),
        (dict(K=0), E), (dict(K=131072), E), (dict(act=2), E), (dict(off=None), E),
        (dict(off=None, E=1), E),                                # counts without offsets
        (dict(ap=128), E), (dict(ap=-16), E), (dict(sp=8), E), (dict(sp=-4), E),
        (dict(ap=2 * moe.MOE_MAX_MX_PITCH), E), (dict(sp=moe.MOE_MAX_MX_PITCH + 4), E),
        (dict(K=272), L), (dict(N=60), L), (dict(N=72, act=1), L), (dict(ap=152), L), (dict(sp=14), L),
        (dict(a=MIS), L), (dict(w=MIS), L), (dict(y=MIS), L), (dict(sa=TWO), L), (dict(sw=TWO), L),
        (dict(off=ODD), L), (dict(cnt=ODD), L)])
    assert moe.lib().moe_expert_matmul_mx(*dict(good, rows=0, a=None).values()) == moe.MOE_OK


def test_scale_rows_are_whole_words():
    assert [moe.mx_scale_bytes(H) for H in (32, 96, 128, 160, 2080, 7168)] == [4, 4, 4, 8, 68, 224]


# ------------------------------------------------------------- marshalling
NAMES = ("moe_balance", "moe_balance_backward", "moe_quantize_mx", "moe_expert_matmul_mx")
T, K = (1 << 33) + 5, 31
LONG = base.LONG | {"seq_len", "q_pitch", "scale_pitch"}


def _prototypes():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(build.INCLUDE, "moe.h")).read(), flags=re.S)
    out = {}
    for name in NAMES + base.NAMES + base.OTHERS:
        args = re.search(rf"\bint {name}\(([^)]*)\);", text).group(1)
        out[name] = [re.match(r"(.*?)(\w+)$", " ".join(a.split())).groups()
                     for a in args.split(",")]
    return out


PROTO = _prototypes()


def _arguments(name):
    """A value of its own for every parameter of a wrapper."""
    kinds = {p: t for t, p in PROTO[name]}
    args = {}
    for i, p in enumerate(inspect.signature(getattr(moe, name)).parameters):
        if p == "stream":
            args[p] = Stream()
        elif p == "workspace" or "*" in kinds[p]:
            args[p] = Buf(0x7F0000000000 + 0x1000 * (i + 1), (T, K) if p == "topk_idx" else None)
        else:
            args[p] = ((1 << 33) if kinds[p].startswith("int64") else 100) + i
    return args


def _expected(name, args):
    out = []
    for _, p in PROTO[name]:
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
    src, so = os.path.join(d, "stub.cpp"), os.path.join(d, "libstub_mx.so")
    with open(src, "w") as f:
        f.write('#include "moe.h"\nextern "C" { unsigned long long rec[32]; int n_rec, code; }\n')
        for name, params in PROTO.items():
            f.write(f'extern "C" int {name}({", ".join(t + p for t, p in params)}) {{\n  n_rec = 0;\n')
            f.write("".join(f"  rec[n_rec++] = (unsigned long long){p};\n" for _, p in params))
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
            return list((ctypes.c_ulonglong * 32).in_dll(lib, "rec"))[:n]

    yield Stub
    calls.init(moe.LIB_PATH, ctypes.ArgumentError, ctypes.c_int, torch._C._cuda_getDevice,
               torch._C._cuda_getCurrentRawStream)


@pytest.mark.parametrize("name", NAMES)
def test_every_argument_arrives(stub, name):
    args = _arguments(name)
    getattr(moe, name)(**args)
    assert stub.recorded() == _expected(name, args)
    for p, v in args.items():
        if isinstance(v, Buf) and p != "topk_idx":
            less = dict(args, **{p: None})
            getattr(moe, name)(**less)
            assert stub.recorded() == _expected(name, less), p


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


def test_host_tensors_are_refused():
    x = torch.zeros(4, 32, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensors"):
        moe.moe_quantize_mx(x, 4, 32, None, None)
