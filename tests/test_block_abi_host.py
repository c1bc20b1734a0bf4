"""The transformer block operators' C ABI without a GPU: exports, struct layouts, stated workspaces, refusals before any
HIP call, and the binding's own checks.  Fake device addresses are never dereferenced."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

import paper_2104_05588_amd as daso
from paper_2104_05588_amd import _block as K
from paper_2104_05588_amd import _lib as L
from paper_2104_05588_amd import build as B
from tests.test_train_abi_host import call, made, need, no_gpu, refused

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "daso_block.h")
A, MB = 0x10000000, 1 << 20
OK, EINVAL, EALIGN, EALIAS, ENOSPACE = L.DASO_OK, L.DASO_EINVAL, L.DASO_EALIGN, L.DASO_EALIAS, L.DASO_ENOSPACE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.LIB_PATH):
        B.build()
    return K._load()


def test_header_and_exports(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"^\s*int\s+(daso_\w+)\s*\(", text, flags=re.M))
    assert names == set(K.EXPORTED_BLOCK)
    for name in names:
        assert hasattr(lib, name), name
    for name, value in re.findall(r"#define (DASO_\w+) (\d+)u?\b", text):
        assert getattr(K, name) == int(value), name


def test_struct_layouts_match_header(tmp_path):
    structs = [K.daso_heads, K.daso_rotary_args, K.daso_attention_args, K.daso_span, K.daso_clip_args]
    src = ["#include <stdio.h>", "#include <stddef.h>", '#include "daso_block.h"', "int main(void) {"]
    for st in structs:
        src.append(f'  printf("{st.__name__} size %zu\\n", sizeof({st.__name__}));')
        src += [f'  printf("{st.__name__} {f[0]} %zu\\n", offsetof({st.__name__}, {f[0]}));' for f in st._fields_]
    c = tmp_path / "layout.c"
    c.write_text("\n".join(src + ["  return 0; }"]) + "\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include", str(c), "-o",
                    str(exe)], check=True)
    found = {st.__name__: st for st in structs}
    lines = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n")
    assert len(lines) > 50
    for line in filter(None, lines):
        st, f, v = line.split()
        assert int(v) == (ctypes.sizeof(found[st]) if f == "size" else getattr(found[st], f).offset), line


def rows(at, token, head):
    return K.daso_heads(at, token, head)


NEVER = (1 << 62, -1, 1 << 60)


def test_rotary_rejects(lib):
    no_gpu()
    h = lambda i, n=4: rows(A + i * MB, n * 64, 64)  # noqa: E731
    base = dict(tokens=10, heads=4, kv_heads=2, dim=64, rotated=64, type=1, eps=1e-6, positions=A + 20 * MB, frequencies=A + 21 * MB,
                q_weight=A + 22 * MB, k_weight=A + 23 * MB, q=h(0), k=h(1, 2), q_out=h(2), k_out=h(3, 2), dq_out=h(4), dk_out=h(5, 2),
                dq=h(6), dk=h(7, 2), dq_weight=A + 24 * MB, dk_weight=A + 25 * MB, workspace=A + 30 * MB, workspace_bytes=MB)
    both = [(dict(tokens=-1), EINVAL), (dict(tokens=(1 << 24) + 1), EINVAL), (dict(heads=0), EINVAL), (dict(kv_heads=0), EINVAL),
            (dict(heads=1025), EINVAL), (dict(dim=60), EINVAL), (dict(dim=136), EINVAL), (dict(dim=0), EINVAL), (dict(rotated=4), EINVAL),
            (dict(rotated=72), EINVAL), (dict(rotated=-8), EINVAL), (dict(type=2), EINVAL), (dict(eps=-1.0), EINVAL),
            (dict(eps=float("nan")), EINVAL), (dict(flags=2), EINVAL), (dict(reserved=1), EINVAL), (dict(q=rows(None, 256, 64)), EINVAL),
            (dict(k=rows(None, 128, 64)), EINVAL), (dict(positions=None), EINVAL),
            (dict(frequencies=None), EINVAL), (dict(positions=A + 20 * MB + 4), EALIGN), (dict(frequencies=A + 21 * MB + 4), EALIGN),
            (dict(q_weight=A + 22 * MB + 2), EALIGN), (dict(q=rows(A + 1, 256, 64)), EALIGN), (dict(q=rows(A, 255, 64)), EINVAL),
            (dict(q=rows(A, 256, 63)), EINVAL), (dict(q=rows(A, 64, 64)), EINVAL), (dict(q=rows(A, 300, 2000)), EINVAL)]
    both += [(dict(q=rows(A, s, 64)), EINVAL) for s in NEVER] + [(dict(k=rows(A + MB, 128, s)), EINVAL) for s in NEVER]
    forward = [(dict(q_out=rows(None, 256, 64)), EINVAL), (dict(q_out=rows(A + 64, 256, 64)), EALIAS), (dict(q_out=rows(A, 320, 64)), EALIAS),
               (dict(q_out=rows(A, 256, 32)), EINVAL), (dict(k_out=rows(A + 2 * MB, 128, 64)), EALIAS), (dict(q_out=rows(A + MB, 256, 64)), EALIAS),
               (dict(k_out=rows(A + 20 * MB, 128, 64)), EALIAS), (dict(q_out=rows(A + 22 * MB, 256, 64)), EALIAS),
               # in place, but a row of it with other distances between the heads
               (dict(tokens=1, q=rows(A, 0, 64), q_out=rows(A, 0, 128)), EALIAS), (dict(tokens=0, q=rows(None, 0, 0), positions=None), OK)]
    refused(lib.daso_head_norm_rotary, K.daso_rotary_args, base, both + forward)
    rc, n = need(lib.daso_head_norm_rotary_backward_workspace, made(K.daso_rotary_args, base))
    assert rc == OK and 0 < n <= MB and n % (2 * 64 * 4) == 0
    backward = [(dict(dq=rows(None, 256, 64)), EINVAL), (dict(dq_out=rows(None, 256, 64)), EINVAL), (dict(dq=rows(A, 256, 64)), EALIAS),
                (dict(dq=rows(A + 4 * MB, 320, 64)), EALIAS), (dict(dk=rows(A + 6 * MB, 128, 64)), EALIAS), (dict(dq_weight=A + 22 * MB), EALIAS),
                (dict(dk_weight=A + 24 * MB + 16), EALIAS), (dict(dq_weight=A + 24 * MB + 1), EALIGN), (dict(dk=rows(A + 5 * MB, 0, 0)), EINVAL),
                (dict(workspace_bytes=n - 1), ENOSPACE), (dict(workspace=None), EINVAL), (dict(workspace=A + 30 * MB + 64), EALIGN),
                (dict(tokens=0, dq_weight=None, dk_weight=None), OK)]
    refused(lib.daso_head_norm_rotary_backward, K.daso_rotary_args, base, both + backward)
    assert need(lib.daso_head_norm_rotary_backward_workspace, made(K.daso_rotary_args, base, tokens=0)) == (OK, 0)
    for fn in (lib.daso_head_norm_rotary, lib.daso_head_norm_rotary_backward, lib.daso_head_norm_rotary_backward_workspace):
        assert fn(None, None) == EINVAL


def test_rotary_in_place_is_of_the_same_distances(lib):
    """With tokens and heads exchanged the same bytes are other tokens' rows: no output may lie so over its input."""
    no_gpu()
    for n, kv in ((4, 4), (7, 7), (3, 2)):
        token, head = (n * 64, 64), (64, n * 64)
        apart = lambda i, s: rows(A + i * MB, *s)  # noqa: E731
        base = dict(tokens=n, heads=n, kv_heads=kv, dim=64, rotated=64, type=1, eps=1e-6, positions=A + 20 * MB, frequencies=A + 21 * MB,
                    q=apart(0, token), k=apart(1, token), q_out=apart(2, token), k_out=apart(3, token), dq_out=apart(4, token),
                    dk_out=apart(5, token), dq=apart(6, token), dk=apart(7, token), dq_weight=A + 24 * MB, workspace=A + 30 * MB,
                    workspace_bytes=0)
        refused(lib.daso_head_norm_rotary, K.daso_rotary_args, base, [
            (dict(q_out=apart(0, head)), EALIAS), (dict(q=apart(0, head), q_out=apart(0, token)), EALIAS), (dict(k_out=apart(1, head)), EALIAS)])
        # in place with the same distances comes as far as a workspace that is too small
        refused(lib.daso_head_norm_rotary_backward, K.daso_rotary_args, base, [
            (dict(dq=apart(4, head)), EALIAS), (dict(dk=apart(5, head)), EALIAS), (dict(dq_out=apart(4, head), dq=apart(4, head)), ENOSPACE),
            (dict(dq=apart(4, token), dk=apart(5, token)), ENOSPACE)])
    # 3 tokens 100 apart, or 2 heads: both are rows of 24 elements 100 apart
    mixed = dict(base, tokens=3, heads=2, kv_heads=1, dim=8, rotated=8, q=rows(A, 100, 16), k=rows(A + MB, 8, 8))
    refused(lib.daso_head_norm_rotary, K.daso_rotary_args, mixed, [(dict(q_out=rows(A, 8, 100)), EALIAS)])


def test_attention_rejects(lib):
    no_gpu()
    h = lambda i, n=4: rows(A + i * MB, n * 64, 64)  # noqa: E731
    base = dict(tokens=10, heads=4, kv_heads=2, dim=64, type=1, sequences=3, flags=1, scale=0.125, offsets=A + 20 * MB, q=h(0), k=h(1, 2),
                v=h(2, 2), out=h(3), lse=A + 21 * MB, dout=h(4), dq=h(5), dk=h(6, 2), dv=h(7, 2), workspace=A + 30 * MB, workspace_bytes=MB)
    both = [(dict(tokens=-1), EINVAL), (dict(tokens=(1 << 24) + 1), EINVAL), (dict(heads=3), EINVAL), (dict(kv_heads=0), EINVAL),
            (dict(heads=2048), EINVAL), (dict(dim=4), EINVAL), (dict(dim=132), EINVAL), (dict(dim=136), EINVAL), (dict(type=3), EINVAL),
            (dict(scale=0.0), EINVAL), (dict(scale=-1.0), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(scale=3e38), EINVAL), (dict(scale=float("nan")), EINVAL),
            (dict(flags=16), EINVAL), (dict(reserved=1), EINVAL), (dict(sequences=-1), EINVAL), (dict(sequences=(1 << 20) + 1), EINVAL),
            (dict(tokens=1 << 24, heads=16, kv_heads=16), EINVAL), (dict(offsets=None), EINVAL), (dict(offsets=A + 20 * MB + 4), EALIGN),
            (dict(q=rows(None, 256, 64)), EINVAL), (dict(v=rows(None, 128, 64)), EINVAL), (dict(out=rows(None, 256, 64)), EINVAL),
            (dict(lse=None), EINVAL), (dict(lse=A + 21 * MB + 2), EALIGN), (dict(k=rows(A + MB + 1, 128, 64)), EALIGN),
            (dict(k=rows(A + MB, 127, 64)), EINVAL), (dict(v=rows(A, 0, 64)), EINVAL), (dict(v=rows(A, 128, 0)), EINVAL), (dict(v=rows(A, (2 << 20) + 8, 64)), EINVAL),
            (dict(tokens=0, q=rows(None, 0, 0)), OK), (dict(sequences=0, offsets=None), OK)]
    both += [(dict(v=rows(A, s, 64)), EINVAL) for s in NEVER] + [(dict(out=rows(A + 3 * MB, 256, s)), EINVAL) for s in NEVER]
    forward = [(dict(out=rows(A, 256, 64)), EALIAS), (dict(out=rows(A + MB + 128, 256, 64)), EALIAS), (dict(lse=A + 3 * MB), EALIAS),
               (dict(lse=A), EALIAS), (dict(out=rows(A + 20 * MB, 256, 64)), EALIAS)]
    refused(lib.daso_attention, K.daso_attention_args, base, both + forward)
    rc, n = need(lib.daso_attention_backward_workspace, made(K.daso_attention_args, base))
    assert rc == OK and n >= 10 * 4 * 4
    backward = [(dict(dout=rows(None, 256, 64)), EINVAL), (dict(dq=rows(None, 256, 64)), EINVAL), (dict(dk=rows(None, 128, 64)), EINVAL),
                (dict(dq=rows(A, 256, 64)), EALIAS), (dict(dq=rows(A + 4 * MB, 256, 64)), EALIAS), (dict(dv=rows(A + 6 * MB, 128, 64)), EALIAS),
                (dict(dv=rows(A + 2 * MB, 128, 64)), EALIAS), (dict(dk=rows(A + 21 * MB, 128, 64)), EALIAS), (dict(dq=rows(A + 3 * MB, 256, 64)), EALIAS),
                (dict(workspace_bytes=n - 1), ENOSPACE), (dict(workspace=None), EINVAL), (dict(workspace=A + 30 * MB + 64), EALIGN)]
    refused(lib.daso_attention_backward, K.daso_attention_args, base, both + backward)
    for fn in (lib.daso_attention, lib.daso_attention_backward, lib.daso_attention_backward_workspace):
        assert fn(None, None) == EINVAL


def test_rows_beside_one_another_do_not_overlap(lib):
    """Parts of one joint buffer, in both orders, come as far as a workspace that is too small."""
    no_gpu()
    base = dict(tokens=10, heads=2, kv_heads=2, dim=64, type=1, sequences=1, flags=0, scale=0.125, out=rows(A + 3 * MB, 128, 64),
                lse=A + 21 * MB, dout=rows(A + 4 * MB, 128, 64), workspace=A + 30 * MB, workspace_bytes=0)
    columns = [rows(A + i * 256, 384, 64) for i in range(3)] + [rows(A + MB + i * 256, 384, 64) for i in range(3)]
    between = [rows(A + i * 128, 384, 192) for i in range(3)] + [rows(A + MB + i * 128, 384, 192) for i in range(3)]
    blocks = [rows(A + i * 128, 192, 1920) for i in range(3)] + [rows(A + MB + i * 128, 192, 1920) for i in range(3)]
    for q, k, v, dq, dk, dv in (columns, between, blocks):
        a = made(K.daso_attention_args, base, q=q, k=k, v=v, dq=dq, dk=dk, dv=dv)
        assert call(lib.daso_attention_backward, a) == ENOSPACE
        a.dv.data += 2  # into the next token's dq
        assert call(lib.daso_attention_backward, a) == EALIAS


def test_clip_rejects(lib):
    no_gpu()

    def grads(*at):
        return (ctypes.c_void_p * len(at))(*at)

    def spans(*of):
        s = (K.daso_span * max(len(of), 1))()
        for to, (start, n) in zip(s, of):
            to.start, to.n = start, n
        return s

    good = grads(A, A + MB)
    base = dict(n=1000, g=2, ntensors=2, grads=good, tensors=spans((0, 10), (20, 980)), out=A + 2 * MB, norm=A + 3 * MB, norms=A + 4 * MB,
                max_norm=1.0, eps=1e-6, workspace=A + 5 * MB, workspace_bytes=MB)
    rc, n = need(lib.daso_clip_gradients_workspace, made(K.daso_clip_args, base))
    assert rc == OK and n == 16
    refused(lib.daso_clip_gradients, K.daso_clip_args, base, [
        (dict(n=-1), EINVAL), (dict(g=0), EINVAL), (dict(g=65), EINVAL), (dict(ntensors=-1), EINVAL), (dict(tensors=None), EINVAL),
        (dict(tensors=spans((0, 10), (9, 5))), EINVAL), (dict(tensors=spans((0, 10), (20, 981))), EINVAL), (dict(tensors=spans((0, -1), (0, 1))), EINVAL),
        (dict(tensors=spans((-1, 5), (10, 1))), EINVAL), (dict(tensors=spans((0, 1), (1 << 62, 1 << 62))), EINVAL), (dict(eps=-1.0), EINVAL),
        (dict(eps=float("inf")), EINVAL), (dict(max_norm=-1.0), EINVAL), (dict(max_norm=float("nan")), EINVAL), (dict(grads=None), EINVAL),
        (dict(grads=grads(A, None)), EINVAL), (dict(grads=grads(A, A + MB + 4)), EALIGN), (dict(out=A + 2 * MB + 8), EALIGN), (dict(norm=None), EINVAL),
        (dict(norm=A + 3 * MB + 2), EALIGN), (dict(norms=A + 4 * MB + 1), EALIGN), (dict(out=A + 16), EALIAS), (dict(norm=A + 100), EALIAS),
        (dict(norms=A + MB), EALIAS), (dict(norm=A + 2 * MB), EALIAS), (dict(norms=A + 3 * MB), EALIAS), (dict(workspace_bytes=n - 1), ENOSPACE),
        (dict(workspace=None), EINVAL), (dict(workspace=A + 5 * MB + 8), EALIGN)])
    assert need(lib.daso_clip_gradients_workspace, made(K.daso_clip_args, base, ntensors=0, tensors=None, n=0)) == (OK, 0)
    assert lib.daso_clip_gradients(None, None) == EINVAL and lib.daso_clip_gradients_workspace(None, None) == EINVAL


def test_binding_rejects_what_is_not_on_the_device():
    x, at = torch.zeros(4, 2, 64), torch.arange(4)
    with pytest.raises(ValueError, match="device tensor"):
        daso.head_norm_rotary(x, x, at, daso.rotary_frequencies(64, device="cpu"))
    with pytest.raises(ValueError, match="device tensor"):
        daso.packed_attention(x, x, x)
    with pytest.raises(ValueError, match="device tensor"):
        daso.clip_gradients([torch.zeros(8)], 1.0)
    with pytest.raises(ValueError, match="needs a gradient"):
        daso.clip_gradients([], 1.0)
    with pytest.raises(ValueError, match="dimensions"):
        daso.packed_attention(x[0], x, x)
    with pytest.raises(ValueError, match="tokens"):
        daso.packed_attention(x, x[:3], x)
    with pytest.raises(ValueError, match="pairs"):
        daso.rotary_frequencies(7, device="cpu")
    f = daso.rotary_frequencies(8, 100.0, device="cpu")
    assert f.dtype == torch.float64 and torch.allclose(f, torch.tensor([1.0, 0.31622777, 0.1, 0.031622777], dtype=torch.float64))
