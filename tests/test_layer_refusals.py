"""The blocks of a decode layer (sifar_cache_append, sifar_paged_attention, sifar_experts)
refuse, on the host and before any device call, what their contracts leave out, and their
binding passes on what it is given. No GPU is used."""
from __future__ import annotations

import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2607_08973_amd as S

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                      "sifar.h")
MB = 1 << 20  # addresses that a refused call never touches
T, HQ, HK, D, PAGES, PAGE = 4, 6, 2, 32, 7, 16
ROW = HK * D
BF = torch.bfloat16


def append_args(**kw):
    a = S.sifar_cache_append_args(
        dtype=S.SIFAR_BF16, tokens=T, q_heads=HQ, kv_heads=HK, head_dim=D, rotary_dim=D,
        interleaved=0, page_size=PAGE, num_pages=PAGES, sequences=T, max_pages=3, rotary_scale=1.0,
        q=MB, q_stride=HQ * D, q_out=2 * MB, q_out_stride=HQ * D, k=3 * MB, k_stride=ROW, v=4 * MB,
        v_stride=ROW, positions=5 * MB, sequence=6 * MB, pages=7 * MB, pages_stride=3,
        inv_freq=8 * MB, k_cache=9 * MB, v_cache=10 * MB, page_stride=PAGE * ROW, slot_stride=ROW,
        head_stride=D)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def attention_args(**kw):
    a = S.sifar_paged_attention_args(
        dtype=S.SIFAR_BF16, tokens=T, q_heads=HQ, kv_heads=HK, head_dim=D, page_size=PAGE,
        num_pages=PAGES, max_pages=300, max_length=4800, window=0, scale=0.5, softcap=0.0, q=MB,
        q_stride=HQ * D, k_cache=2 * MB, v_cache=3 * MB, page_stride=PAGE * ROW, slot_stride=ROW,
        head_stride=D, pages=4 * MB, pages_stride=300, lengths=5 * MB, sinks=6 * MB, out=7 * MB,
        out_stride=HQ * D, lse=8 * MB, workspace=16 * MB,
        workspace_bytes=S.load().sifar_paged_attention_workspace(T, HQ, HK, D, 4800))
    for k, v in kw.items():
        setattr(a, k, v)
    return a


H, I, E, K = 64, 48, 5, 3


def experts_args(**kw):
    a = S.sifar_experts_args(
        dtype=S.SIFAR_BF16, tokens=T, hidden=H, inter=I, experts=E, topk=K, first_expert=0,
        activation=0, x=MB, x_stride=H, ids=2 * MB, weights=3 * MB, w_in=4 * MB,
        w_in_stride=2 * I * H, w_out=5 * MB, w_out_stride=I * H, out=6 * MB, out_stride=H,
        workspace=7 * MB, workspace_bytes=S.load().sifar_experts_workspace(T, K, I))
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD_APPEND = [
    dict(dtype=3), dict(dtype=-1), dict(tokens=-1), dict(tokens=S.SIFAR_ROWS_MAX_TOKENS + 1),
    dict(q_heads=-1), dict(q_heads=1025), dict(kv_heads=0), dict(kv_heads=1025), dict(head_dim=0),
    dict(head_dim=36), dict(head_dim=264), dict(rotary_dim=-2), dict(rotary_dim=34),
    dict(rotary_dim=31), dict(interleaved=2), dict(interleaved=-1), dict(page_size=0),
    dict(page_size=65537), dict(num_pages=0), dict(sequences=0), dict(max_pages=0),
    dict(sequence=None, sequences=T - 1), dict(q=None), dict(q_out=None), dict(q_heads=0),
    dict(k=None), dict(v=None), dict(positions=None), dict(pages=None), dict(inv_freq=None),
    dict(rotary_dim=0), dict(k_cache=None), dict(v_cache=None), dict(q=MB + 8), dict(q_out=2 * MB + 8),
    dict(k=3 * MB + 2), dict(v=4 * MB + 8), dict(k_cache=9 * MB + 8), dict(v_cache=10 * MB + 8),
    dict(positions=5 * MB + 2), dict(sequence=6 * MB + 1), dict(pages=7 * MB + 2),
    dict(inv_freq=8 * MB + 2), dict(q_stride=HQ * D - 8), dict(q_stride=HQ * D + 4),
    dict(q_out_stride=0), dict(k_stride=ROW - 8), dict(k_stride=-ROW), dict(v_stride=ROW + 4),
    dict(pages_stride=-1), dict(pages_stride=1 << 40), dict(sequences=2 ** 31 - 1, pages_stride=1 << 12),
    dict(page_stride=PAGE * ROW - 8), dict(slot_stride=ROW - 8),
    dict(slot_stride=ROW + 4), dict(head_stride=D - 8), dict(head_stride=-D), dict(page_stride=0),
    dict(page_stride=1 << 41),
    # outputs over outputs and inputs
    dict(v_cache=9 * MB), dict(v_cache=9 * MB + 2 * D), dict(v_cache=9 * MB + 2 * ROW),
    dict(k_cache=10 * MB + 2 * (PAGES * PAGE - 1) * ROW), dict(q_out=MB + 2 * D),
    dict(q_out=MB, q_out_stride=2 * HQ * D), dict(q_out=3 * MB), dict(q_out=4 * MB - 16),
    dict(q_out=9 * MB), dict(k=9 * MB), dict(v=10 * MB + 2 * ROW), dict(q=9 * MB, q_out=9 * MB),
    dict(positions=9 * MB), dict(pages=10 * MB), dict(inv_freq=2 * MB), dict(sequence=2 * MB),
]
BAD_ATTENTION = [
    dict(dtype=3), dict(tokens=-1), dict(tokens=S.SIFAR_ATTENTION_MAX_TOKENS + 1), dict(q_heads=0),
    dict(q_heads=5), dict(q_heads=1026), dict(kv_heads=0), dict(kv_heads=-2), dict(head_dim=0),
    dict(head_dim=20), dict(head_dim=264), dict(page_size=0), dict(page_size=65537),
    dict(num_pages=0), dict(max_pages=0), dict(max_length=0), dict(max_length=(1 << 24) + 1),
    dict(window=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(softcap=-1.0),
    dict(softcap=float("nan")), dict(softcap=float("inf")), dict(q=None), dict(k_cache=None),
    dict(v_cache=None), dict(pages=None), dict(lengths=None), dict(out=None), dict(workspace=None),
    dict(q=MB + 8), dict(k_cache=2 * MB + 8), dict(v_cache=3 * MB + 8), dict(out=7 * MB + 8),
    dict(workspace=16 * MB + 8), dict(pages=4 * MB + 2), dict(lengths=5 * MB + 1),
    dict(sinks=6 * MB + 2), dict(lse=8 * MB + 2), dict(q_stride=HQ * D - 8),
    dict(q_stride=HQ * D + 4), dict(out_stride=0), dict(page_stride=PAGE * ROW - 8),
    dict(slot_stride=ROW + 4), dict(head_stride=0), dict(pages_stride=-1), dict(pages_stride=1 << 40),
    dict(workspace_bytes=attention_args().workspace_bytes - 1), dict(workspace_bytes=-1),
    dict(out=MB + 2 * D), dict(out=MB, out_stride=2 * HQ * D), dict(out=2 * MB), dict(out=4 * MB),
    dict(out=5 * MB), dict(out=6 * MB), dict(out=8 * MB), dict(out=16 * MB), dict(lse=16 * MB),
    dict(lse=MB), dict(lse=2 * MB), dict(workspace=MB), dict(workspace=3 * MB), dict(workspace=4 * MB),
]
BAD_EXPERTS = [
    dict(dtype=3), dict(tokens=-1), dict(tokens=129), dict(tokens=128, topk=9), dict(hidden=0),
    dict(hidden=12), dict(hidden=65544), dict(inter=0), dict(inter=20), dict(inter=65544),
    dict(experts=0), dict(experts=1025), dict(topk=0), dict(topk=33), dict(first_expert=-1),
    dict(first_expert=2 ** 31 - 1), dict(first_expert=2 ** 31 - E),
    dict(activation=2), dict(activation=-1), dict(x=None), dict(ids=None), dict(weights=None),
    dict(w_in=None), dict(w_out=None), dict(out=None), dict(workspace=None), dict(x=MB + 8),
    dict(w_in=4 * MB + 8), dict(w_out=5 * MB + 8), dict(out=6 * MB + 8), dict(workspace=7 * MB + 8),
    dict(ids=2 * MB + 2), dict(weights=3 * MB + 1), dict(x_stride=H - 8), dict(x_stride=H + 4),
    dict(out_stride=0), dict(w_in_stride=2 * I * H - 8), dict(w_out_stride=I * H + 4),
    dict(w_out_stride=-I * H), dict(workspace_bytes=experts_args().workspace_bytes - 1),
    dict(out=MB), dict(out=2 * MB), dict(out=3 * MB), dict(out=4 * MB), dict(out=5 * MB + 2 * H),
    dict(out=7 * MB), dict(workspace=MB), dict(workspace=2 * MB), dict(workspace=4 * MB),
    dict(workspace=5 * MB + 16),
]
CASES = ([("sifar_cache_append", append_args, kw) for kw in BAD_APPEND]
         + [("sifar_paged_attention", attention_args, kw) for kw in BAD_ATTENTION]
         + [("sifar_experts", experts_args, kw) for kw in BAD_EXPERTS])


@pytest.mark.parametrize("fn,args,kw", CASES, ids=lambda v: ",".join(
    f"{k}={x}" for k, x in v.items()) if isinstance(v, dict) else getattr(v, "__name__", v))
def test_refused_by_the_library(fn, args, kw):
    assert getattr(S.load(), fn)(ctypes.byref(args(**kw)), None) == S.SIFAR_EINVAL


def test_null_and_empty_calls():
    L = S.load()
    for fn, args in (("sifar_cache_append", append_args), ("sifar_paged_attention", attention_args),
                     ("sifar_experts", experts_args)):
        assert getattr(L, fn)(None, None) == S.SIFAR_EINVAL
        a = args(tokens=0)
        for name, kind in a._fields_:
            if kind is ctypes.c_void_p:
                setattr(a, name, None)
        assert getattr(L, fn)(ctypes.byref(a), None) == S.SIFAR_OK, fn


@pytest.mark.parametrize("name", ["sifar_cache_append_args", "sifar_paged_attention_args",
                                  "sifar_experts_args"])
def test_layout_matches_a_c_compiler(name, tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    cls = getattr(S, name)
    body = re.search(r"typedef struct \{([^{}]*)\} " + name + ";", open(HEADER).read()).group(1)
    assert re.findall(r"\b(\w+);", body) == [f for f, _ in cls._fields_]
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "sifar.h"', "int main(void) {",
             f'    printf("size %zu\\n", sizeof({name}));']
    lines += [f'    printf("{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["    return 0;", "}"]) + "\n")
    subprocess.run([cc, "-std=c11", "-I", os.path.dirname(HEADER), str(src), "-o", str(exe)],
                   check=True)
    for line in subprocess.run([str(exe)], check=True, capture_output=True,
                               text=True).stdout.split("\n")[:-1]:
        what, value = line.split()
        assert int(value) == (ctypes.sizeof(cls) if what == "size" else getattr(cls, what).offset)


# ---- workspaces --------------------------------------------------------------------------------

def test_workspaces_grow():
    w = S.sifar_paged_attention_workspace
    assert w(0, 8, 2, 64, 4096) == 0 and w(64, 8, 2, 64, 100) == 0
    for heads, kv, dim in ((32, 8, 128), (1, 1, 8), (34, 1, 256), (1024, 1024, 64)):
        for length in (1, 257, 1000, 5000, 131072, 1 << 24):
            sizes = [w(t, heads, kv, dim, length) for t in (1, 2, 3, 7, 63, 64, 65, 255, 4096, 32768)]
            assert sizes == sorted(sizes), (heads, length)
        for tokens in (1, 5, 64, 300):
            sizes = [w(tokens, heads, kv, dim, n) for n in (
                1, 128, 256, 257, 511, 2048, 2049, 4097, 100000, 131072, 1 << 20, 1 << 24)]
            assert sizes == sorted(sizes), (heads, tokens)
    e = S.sifar_experts_workspace
    assert e(1, 8, 768) >= 8 * 768 * 4 and e(128, 8, 64) >= e(127, 8, 64) >= e(127, 7, 64)


@pytest.mark.parametrize("call", [
    lambda: S.sifar_paged_attention_workspace(-1, 8, 2, 64, 100),
    lambda: S.sifar_paged_attention_workspace(1, 7, 2, 64, 100),
    lambda: S.sifar_paged_attention_workspace(1, 8, 2, 60, 100),
    lambda: S.sifar_paged_attention_workspace(1, 8, 2, 64, 0),
    lambda: S.sifar_paged_attention_workspace((1 << 32) + 1, 8, 2, 64, 100),
    lambda: S.sifar_paged_attention_workspace(1, 8, 2, 64, 1 << 40),
    lambda: S.sifar_experts_workspace(129, 1, 64), lambda: S.sifar_experts_workspace(1, 33, 64),
    lambda: S.sifar_experts_workspace(1, 1, 60), lambda: S.sifar_experts_workspace(1 << 32, 1, 64),
    lambda: S.sifar_experts_workspace(1, 1.5, 64),
])
def test_workspaces_refused(call):
    with pytest.raises(S.SifarError) as e:
        call()
    assert e.value.code == S.SIFAR_EINVAL


# ---- the binding -------------------------------------------------------------------------------

class Recorder:
    """Stands in for the library where host tensors play device tensors."""

    def __init__(self):
        self.calls = []

    def sifar_cache_append(self, packed, stream):
        self.calls.append(S.sifar_cache_append_args.from_buffer_copy(packed))
        return 0

    def sifar_paged_attention(self, packed, stream):
        self.calls.append(S.sifar_paged_attention_args.from_buffer_copy(packed))
        return 0

    def sifar_experts(self, packed, stream):
        self.calls.append(S.sifar_experts_args.from_buffer_copy(packed))
        return 0

    def sifar_strerror(self, code):
        return b""


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(S, "_lib", r)
    monkeypatch.setattr(S, "_gpu", lambda fn, name, t: -1)   # a host tensor's device
    monkeypatch.setattr(S, "_row_stream", lambda stream, dev: 0)
    return r


def z(*s, dt=BF):
    return torch.zeros(*s, dtype=dt)


def i32(*s):
    return torch.zeros(*s, dtype=torch.int32)


def append_tensors(**kw):
    x = z(T, HQ + 2 * HK, D)
    a = dict(k=x[:, HQ:HQ + HK], v=x[:, HQ + HK:], positions=i32(T), pages=i32(T, 3),
             k_cache=z(PAGES, PAGE, HK, D), v_cache=z(PAGES, PAGE, HK, D), q=x[:, :HQ],
             q_out=z(T, HQ, D), inv_freq=torch.zeros(D // 2), sequence=i32(T))
    a.update(kw)
    return a


def attention_tensors(**kw):
    a = dict(q=z(T, HQ, D), k_cache=z(PAGES, HK, PAGE, D).transpose(1, 2),
             v_cache=z(PAGES, HK, PAGE, D).transpose(1, 2), pages=i32(T, 5)[:, :4], lengths=i32(T),
             out=z(T, HQ, D), workspace=torch.zeros(100, dtype=torch.uint8),
             sinks=torch.zeros(HQ), lse=torch.zeros(T, HQ))
    a.update(kw)
    return a


def experts_tensors(**kw):
    a = dict(x=z(T, 2 * H)[:, :H], ids=i32(T, K), weights=torch.zeros(T, K), w_in=z(E, 2 * I, H),
             w_out=z(E, H, I), out=z(T, H), workspace=torch.zeros(99, dtype=torch.uint8))
    a.update(kw)
    return a


def test_append_marshalling(recorder):
    t = append_tensors()
    S.sifar_cache_append(**t, interleaved=True, rotary_scale=0.5)
    c = recorder.calls[0]
    assert (c.dtype, c.tokens, c.q_heads, c.kv_heads, c.head_dim, c.rotary_dim, c.interleaved,
            c.page_size, c.num_pages, c.sequences, c.max_pages, c.rotary_scale) == (
        S.SIFAR_BF16, T, HQ, HK, D, D, 1, PAGE, PAGES, T, 3, 0.5)
    for name in ("k", "v", "positions", "pages", "k_cache", "v_cache", "q", "q_out", "inv_freq",
                 "sequence"):
        assert getattr(c, name) == t[name].data_ptr(), name
    wide = (HQ + 2 * HK) * D
    assert (c.q_stride, c.q_out_stride, c.k_stride, c.v_stride, c.pages_stride, c.page_stride,
            c.slot_stride, c.head_stride) == (wide, HQ * D, wide, wide, 3, PAGE * ROW, ROW, D)
    S.sifar_cache_append(**append_tensors(q=None, q_out=None, inv_freq=None, sequence=None))
    c = recorder.calls[1]
    assert (c.q, c.q_out, c.inv_freq, c.sequence, c.q_heads, c.rotary_dim, c.interleaved,
            c.rotary_scale) == (None, None, None, None, 0, 0, 0, 1.0)


def test_attention_marshalling(recorder):
    t = attention_tensors()
    S.sifar_paged_attention(**t, max_length=50, scale=0.25, window=7, softcap=30.0)
    c = recorder.calls[0]
    assert (c.dtype, c.tokens, c.q_heads, c.kv_heads, c.head_dim, c.page_size, c.num_pages,
            c.max_pages, c.max_length, c.window, c.scale, c.softcap, c.workspace_bytes) == (
        S.SIFAR_BF16, T, HQ, HK, D, PAGE, PAGES, 4, 50, 7, 0.25, 30.0, 100)
    for name in ("q", "k_cache", "v_cache", "pages", "lengths", "out", "workspace", "sinks", "lse"):
        assert getattr(c, name) == t[name].data_ptr(), name
    assert (c.q_stride, c.out_stride, c.pages_stride, c.page_stride, c.slot_stride,
            c.head_stride) == (HQ * D, HQ * D, 5, PAGE * ROW, D, PAGE * D)
    S.sifar_paged_attention(**attention_tensors(workspace=None, sinks=None, lse=None))
    c = recorder.calls[1]
    assert (c.workspace, c.workspace_bytes, c.sinks, c.lse, c.max_length, c.window, c.softcap) == (
        None, 0, None, None, 4 * PAGE, 0, 0.0)
    assert abs(c.scale - D ** -0.5) < 1e-8


def test_experts_marshalling(recorder):
    t = experts_tensors()
    S.sifar_experts(**t, activation="gelu", first_expert=10)
    c = recorder.calls[0]
    assert (c.dtype, c.tokens, c.hidden, c.inter, c.experts, c.topk, c.first_expert, c.activation,
            c.workspace_bytes) == (S.SIFAR_BF16, T, H, I, E, K, 10, 1, 99)
    for name in ("x", "ids", "weights", "w_in", "w_out", "out", "workspace"):
        assert getattr(c, name) == t[name].data_ptr(), name
    assert (c.x_stride, c.w_in_stride, c.w_out_stride, c.out_stride) == (2 * H, 2 * I * H, I * H, H)


BAD_BINDING = [
    ("append", kw) for kw in (
        dict(k=None), dict(v=None), dict(positions=None), dict(pages=None), dict(k_cache=None),
        dict(v_cache=None), dict(q=None), dict(q_out=None), dict(k=z(T, ROW)),
        dict(k=z(T, HK, D).float()), dict(k=z(T, HK, 2 * D)[..., ::2]),
        dict(k=z(T, D, HK).transpose(1, 2)), dict(v=z(T, HK + 1, D)), dict(v=z(T, 2 * HK, D)[:, ::2]),
        dict(k=z(T, HK, D, dt=torch.float64)), dict(q=z(T + 1, HQ, D)), dict(q=z(T, HQ, D + 8)),
        dict(q_out=z(T, HQ + 1, D)), dict(q=z(T, HQ, D).float()), dict(positions=i32(T).long()),
        dict(positions=i32(T + 1)), dict(sequence=i32(T, 1)), dict(pages=i32(T)),
        dict(pages=i32(T, 6)[:, ::2]), dict(pages=torch.zeros(T, 3)), dict(inv_freq=torch.zeros(0)),
        dict(inv_freq=torch.zeros(129)), dict(inv_freq=z(D // 2)), dict(k_cache=z(PAGES, PAGE, ROW)),
        dict(k_cache=z(PAGES, PAGE, HK + 1, D)), dict(v_cache=z(PAGES, PAGE, 2 * HK, D)[:, :, ::2]),
        dict(v_cache=z(PAGES, PAGE, HK, D).float()), dict(rotary_scale=1e39),
        dict(rotary_scale=None))
] + [
    ("attention", kw) for kw in (
        dict(q=None), dict(k_cache=None), dict(v_cache=None), dict(pages=None), dict(lengths=None),
        dict(out=None), dict(q=z(T, HQ * D)), dict(q=z(T, HQ, D).float()), dict(out=z(T, HQ, D + 8)),
        dict(q=z(T, HQ, D, dt=torch.float64)), dict(k_cache=z(PAGES, PAGE, HK, D)),
        dict(pages=i32(T + 1, 4)), dict(lengths=i32(T + 1)), dict(lengths=i32(T).long()),
        dict(sinks=z(HQ)), dict(sinks=torch.zeros(HK)), dict(lse=torch.zeros(T, HQ + 1)[:, :HQ]),
        dict(lse=z(T, HQ)), dict(workspace=torch.zeros(100)), dict(workspace=torch.zeros(
            10, 10, dtype=torch.uint8)), dict(max_length=1 << 31), dict(window=1 << 31),
        dict(scale=1e39), dict(softcap="x"), dict(window=1.5))
] + [
    ("experts", kw) for kw in (
        dict(x=None), dict(ids=None), dict(weights=None), dict(w_in=None), dict(w_out=None),
        dict(out=None), dict(workspace=None), dict(x=z(H)), dict(x=z(T, H, dt=torch.float64)),
        dict(x=z(T, H).float()), dict(ids=i32(T + 1, K)), dict(ids=i32(T, K).long()),
        dict(ids=i32(T, 2 * K)[:, :K]), dict(weights=z(T, K)), dict(weights=torch.zeros(T, K + 1)),
        dict(w_in=z(E, I, H)), dict(w_in=z(E, H, 2 * I).transpose(1, 2)), dict(w_in=z(E + 1, 2 * I, H)),
        dict(w_out=z(E, H)), dict(w_out=z(E, H + 8, I)), dict(out=z(T, H + 8)),
        dict(workspace=torch.zeros(99)), dict(activation="relu"), dict(activation=2),
        dict(first_expert=1 << 31), dict(first_expert=None))
]


@pytest.mark.parametrize("op,kw", BAD_BINDING, ids=range(len(BAD_BINDING)))
def test_refused_by_the_binding(recorder, op, kw):
    call, tensors = {"append": (S.sifar_cache_append, append_tensors),
                     "attention": (S.sifar_paged_attention, attention_tensors),
                     "experts": (S.sifar_experts, experts_tensors)}[op]
    with pytest.raises(S.SifarError) as e:
        call(**tensors(**kw))
    assert e.value.code == S.SIFAR_EINVAL and not recorder.calls


def test_host_tensors_are_refused():
    for call, tensors in ((S.sifar_cache_append, append_tensors()),
                          (S.sifar_paged_attention, attention_tensors()),
                          (S.sifar_experts, experts_tensors())):
        with pytest.raises(S.SifarError) as e:
            call(**tensors)
        assert e.value.code == S.SIFAR_EINVAL
