"""CPU checks of the packed-sequence operators: exports, documented refusals,
workspace sizes, the host layer under sanitizers, and the wait states around
the attention kernels' asm statements."""

import os
import shutil
import subprocess

import pytest

import test_asm_wait_states as waits
from conftest import device_asm
from paper_2606_10415_amd import lt

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x1000_0000   # aligned address that is never dereferenced (host-side rejection)
INV, UNS, WS = lt.LT_ERR_INVALID_ARG, lt.LT_ERR_UNSUPPORTED, lt.LT_ERR_WORKSPACE


def test_declared_and_exported():
    names = {"lt_attn_mod_fwd", "lt_attn_mod_bwd", "lt_attn_mod_bwd_workspace_size", "lt_qknorm_rope_fwd",
             "lt_qknorm_rope_bwd", "lt_qknorm_rope_bwd_workspace_size", "lt_embed_fwd", "lt_embed_bwd",
             "lt_embed_bwd_workspace_size"}
    assert names <= set(lt.declared_functions())
    for n in names:
        assert hasattr(lt._lib, n) and hasattr(lt, n), n


def status(f, a, **kw):
    a = dict(a, **kw)
    try:
        f(**a)
    except lt.LtError as e:
        assert lt.last_error() != ""
        return e.status
    return lt.LT_OK


FWD = dict(Q=FAKE, K=FAKE, V=FAKE, q_row_stride=384, kv_row_stride=384, O=FAKE, o_row_stride=128, LSE=FAKE, LO=FAKE,
           HI=None, slopes=None, cap=0.0, B=1, S=16, Hq=2, Hkv=1, D=64, scale=0.125, causal=1, stream=0)


@pytest.mark.parametrize("kw,st", [
    (dict(Q=None), INV), (dict(O=None), INV), (dict(LSE=None), INV), (dict(S=0), INV), (dict(B=0), INV),
    (dict(Hq=3, Hkv=2, q_row_stride=800, kv_row_stride=800, o_row_stride=800), INV), (dict(causal=2), INV),
    (dict(scale=0.0), INV), (dict(scale=float("inf")), INV), (dict(cap=-1.0), INV), (dict(cap=float("nan")), INV),
    (dict(cap=float("inf")), INV), (dict(q_row_stride=64), INV), (dict(kv_row_stride=32), INV),
    (dict(o_row_stride=64), INV), (dict(cap=1001.0), UNS), (dict(cap=1e-38, scale=10.0), UNS), (dict(D=32), UNS),
    (dict(D=96, o_row_stride=192), UNS), (dict(S=(1 << 19) + 1), UNS), (dict(q_row_stride=388), UNS), (dict(kv_row_stride=1 << 22), UNS),
    (dict(o_row_stride=1 << 22), UNS), (dict(K=FAKE + 8), UNS), (dict(O=FAKE + 2), UNS), (dict(LO=FAKE + 2), UNS),
    (dict(HI=FAKE + 1), UNS), (dict(slopes=FAKE + 2), UNS), (dict(B=1 << 27, S=1 << 19), UNS),
    (dict(B=1 << 22, S=1), UNS),
])
def test_attention_refusals(kw, st):
    assert status(lt.lt_attn_mod_fwd, FWD, **kw) == st
    n = lt.lt_attn_mod_bwd_workspace_size(1, 16, 2, 1, 64, 1)
    back = dict(FWD, dO=FAKE, dQ=FAKE, dK=FAKE, dV=FAKE, dq_row_stride=384, dkv_row_stride=384, workspace=FAKE,
                ws_bytes=n)
    assert status(lt.lt_attn_mod_bwd, back, **kw) == st


@pytest.mark.parametrize("kw,st", [
    (dict(dO=None), INV), (dict(dV=None), INV), (dict(dq_row_stride=64), INV), (dict(dkv_row_stride=8), INV),
    (dict(dq_row_stride=388), UNS), (dict(dkv_row_stride=1 << 22), UNS), (dict(dK=FAKE + 8), UNS),
    (dict(workspace=None), WS), (dict(ws_bytes=0), WS), (dict(workspace=FAKE + 128), WS),
])
def test_attention_backward_refusals(kw, st):
    n = lt.lt_attn_mod_bwd_workspace_size(1, 16, 2, 1, 64, 1)
    back = dict(FWD, dO=FAKE, dQ=FAKE, dK=FAKE, dV=FAKE, dq_row_stride=384, dkv_row_stride=384, workspace=FAKE,
                ws_bytes=n)
    assert status(lt.lt_attn_mod_bwd, back, **kw) == st
    assert status(lt.lt_attn_mod_bwd, back, ws_bytes=n - 1) == WS


NORM = dict(X=FAKE, ldx=512, Wq=FAKE, Wk=FAKE, CS=FAKE, P=64, POS=None, RSTD=FAKE, B=2, S=32, Hq=3, Hkv=1, D=128,
            stream=0)


@pytest.mark.parametrize("kw,st", [
    (dict(X=None), INV), (dict(Wk=None), INV), (dict(CS=None), INV), (dict(RSTD=None), INV), (dict(B=0), INV),
    (dict(Hkv=0), INV), (dict(P=0), INV), (dict(S=65), INV), (dict(ldx=504), INV), (dict(D=120, ldx=480), UNS),
    (dict(D=272, ldx=1088), UNS), (dict(ldx=516), UNS), (dict(Wq=FAKE + 8), UNS), (dict(CS=FAKE + 4), UNS),
    (dict(POS=FAKE + 2), UNS), (dict(RSTD=FAKE + 2), UNS), (dict(B=1 << 30, S=64), UNS), (dict(B=1 << 20, S=33), UNS),
])
def test_qknorm_refusals(kw, st):
    big = dict(ldy=2048) if kw.get("D", 0) > 128 else dict(ldy=512)
    assert status(lt.lt_qknorm_rope_fwd, dict(NORM, Y=FAKE, eps=1e-6, **big), **kw) == st
    n = lt.lt_qknorm_rope_bwd_workspace_size(2, 32, 3, 1, 128)
    back = dict(NORM, dY=FAKE, lddy=2048, dX=FAKE, lddx=big["ldy"], dWq=FAKE, dWk=FAKE, workspace=FAKE, ws_bytes=n)
    assert status(lt.lt_qknorm_rope_bwd, back, **kw) == st


def test_qknorm_further_refusals():
    f = dict(NORM, Y=FAKE, ldy=512, eps=1e-6)
    for kw, st in ((dict(eps=-1.0), INV), (dict(eps=float("nan")), INV), (dict(Y=None), INV), (dict(ldy=8), INV),
                   (dict(Y=FAKE + 8), UNS), (dict(ldy=520), INV)):
        assert status(lt.lt_qknorm_rope_fwd, f, **kw) == st
    n = lt.lt_qknorm_rope_bwd_workspace_size(2, 32, 3, 1, 128)
    b = dict(NORM, dY=FAKE, lddy=512, dX=FAKE, lddx=512, dWq=FAKE, dWk=FAKE, workspace=FAKE, ws_bytes=n)
    for kw, st in ((dict(dY=None), INV), (dict(dWq=None), INV), (dict(lddy=8), INV), (dict(lddy=516), UNS), (dict(lddy=520), INV),
                   (dict(dWk=FAKE + 1), UNS), (dict(workspace=None), WS), (dict(ws_bytes=n - 1), WS)):
        assert status(lt.lt_qknorm_rope_bwd, b, **kw) == st


EMB = dict(ids=FAKE, scale=1.0, T=10, H=64, V=100, stream=0)


@pytest.mark.parametrize("kw,st", [
    (dict(ids=None), INV), (dict(T=-1), INV), (dict(H=0), INV), (dict(V=0), INV), (dict(scale=float("inf")), INV),
    (dict(H=60), UNS), (dict(T=1 << 30), UNS), (dict(V=1 << 30), UNS), (dict(ids=FAKE + 4), UNS),
])
def test_embedding_refusals(kw, st):
    assert status(lt.lt_embed_fwd, dict(EMB, W=FAKE, ldw=64, Y=FAKE, ldy=64), **kw) == st
    n = lt.lt_embed_bwd_workspace_size(10, 64, 100)
    b = dict(EMB, dY=FAKE, lddy=64, accumulate=0, dW=FAKE, lddw=64, workspace=FAKE, ws_bytes=n)
    assert status(lt.lt_embed_bwd, b, **kw) == st


def test_embedding_further_refusals():
    f = dict(EMB, W=FAKE, ldw=64, Y=FAKE, ldy=64)
    for kw, st in ((dict(W=None), INV), (dict(Y=None), INV), (dict(ldw=56), INV), (dict(ldy=68), UNS),
                   (dict(W=FAKE + 8), UNS), (dict(H=65544, ldw=65544, ldy=65544), UNS), (dict(T=0, ids=None), 0)):
        assert status(lt.lt_embed_fwd, f, **kw) == st
    n = lt.lt_embed_bwd_workspace_size(10, 64, 100)
    b = dict(EMB, dY=FAKE, lddy=64, accumulate=0, dW=FAKE, lddw=64, workspace=FAKE, ws_bytes=n)
    for kw, st in ((dict(dY=None), INV), (dict(dW=None), INV), (dict(accumulate=2), INV), (dict(lddw=8), INV),
                   (dict(lddy=68), UNS), (dict(workspace=None), WS), (dict(ws_bytes=0), WS),
                   (dict(T=0, ids=None, dY=None, accumulate=1), 0)):
        assert status(lt.lt_embed_bwd, b, **kw) == st


def test_workspace_sizes():
    up = lambda x: -(-x // 256) * 256

    def attn(B, S, Hq, Hkv, D, causal, chunk, nsplit):
        n32 = -(-S // 32)
        blocks = n32 * (n32 + 1) // 2 if causal else n32 * n32
        return (2 * up(4 * B * Hq * S) + up(8 * B * S) + up(16 * B * n32) + up(16 * B * Hq * -(-S // 128)) +
                up(chunk * (Hq // Hkv) * blocks * 2048) +
                up(B * Hq * blocks) +
                (up(8 * chunk * nsplit * S * D) if nsplit > 1 else 0))
    # enough key tiles: one chunk, no shares; short sequences of few heads: shares, or not
    assert lt.lt_attn_mod_bwd_workspace_size(1, 4096, 32, 32, 128, 1) == attn(1, 4096, 32, 32, 128, 1, 32, 1)
    assert lt.lt_attn_mod_bwd_workspace_size(1, 2048, 40, 8, 128, 1) == attn(1, 2048, 40, 8, 128, 1, 8, 4)
    assert lt.lt_attn_mod_bwd_workspace_size(4, 333, 16, 16, 64, 0) == attn(4, 333, 16, 16, 64, 0, 64, 1)
    # 8.6 GB of dS blocks: two chunks of eight pairs
    assert lt.lt_attn_mod_bwd_workspace_size(2, 8192, 64, 8, 128, 1) == attn(2, 8192, 64, 8, 128, 1, 8, 2)
    # 128k tokens: a pair at a time, whatever it takes
    assert lt.lt_attn_mod_bwd_workspace_size(1, 131072, 8, 8, 128, 1) == attn(1, 131072, 8, 8, 128, 1, 1, 1)
    for bad in ((0, 16, 2, 1, 64, 1), (1, 16, 3, 2, 64, 1), (1, 16, 2, 1, 96, 1), (1, 16, 2, 1, 64, 2),
                (1, (1 << 19) + 1, 2, 1, 64, 1)):
        assert lt.lt_attn_mod_bwd_workspace_size(*bad) == 0
    assert lt.lt_qknorm_rope_bwd_workspace_size(1, 10, 2, 1, 120) == 0
    assert lt.lt_embed_bwd_workspace_size(10, 60, 100) == 0


def test_wrong_array_types():
    torch = pytest.importorskip("torch")
    for kw in (dict(LO=torch.zeros(16, dtype=torch.int64)), dict(HI=torch.zeros(16)),
               dict(slopes=torch.zeros(2, dtype=torch.float16)), dict(LO=torch.zeros(16, dtype=torch.int32))):
        with pytest.raises(TypeError):               # the last: a host tensor
            lt.lt_attn_mod_fwd(**dict(FWD, **kw))
    with pytest.raises(TypeError):
        lt.lt_embed_fwd(**dict(EMB, ids=torch.zeros(10, dtype=torch.int32), W=FAKE, ldw=64, Y=FAKE, ldy=64))


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include/hip"),
                    reason="needs g++ and the HIP headers")
def test_host_layer_under_sanitizers(tmp_path):
    exe = tmp_path / "packed_host_check"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", f"-I{ROOT}/include",
           os.path.join(ROOT, "paper_2606_10415_amd", "csrc", "packed_api.cpp"),
           os.path.join(ROOT, "tests", "packed_host_check.cpp"), "-L/opt/rocm/lib", "-lamdhip64",
           "-Wl,-rpath,/opt/rocm/lib", "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([str(exe), "20000"], capture_output=True, text=True, env=env, timeout=600)
    print(r.stdout)
    assert r.returncode == 0, (r.stdout[-2000:], r.stderr[-6000:])


@pytest.mark.parametrize("source", ["attn_mod_fwd.hip", "attn_mod_bwd.hip"])
def test_wait_states_of_the_attention_kernels(source):
    kernels = waits.functions(device_asm(source))
    assert sum(len(waits.lds_loads(b)) for b in kernels.values()) > 50
    for early in (waits.early_m0, waits.early_scalars, waits.early_operands):
        bad = [(name[:80], x) for name, blocks in kernels.items() for x in early(blocks)]
        assert not bad, (early.__name__, len(bad), bad[:3])


@pytest.mark.parametrize("source", ["attn_mod_fwd.hip", "attn_mod_bwd.hip", "qknorm_rope.hip", "embed.hip"])
def test_no_packed_fp32_instructions(source):
    assert not [t for t in device_asm(source) if "v_pk_" in t and "_f32" in t and "cvt" not in t][:3]
