"""Host-side checks of the serving operators: exported symbols, refusals before any GPU call, the reference itself."""
import ctypes
import os
import re
import struct
import subprocess

import numpy as np
import pytest
import torch

from oracle import sol_cache_oracle as ora
from paper_2607_24027_amd import binding as sb
from paper_2607_24027_amd import cache as sc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "sol_cache.h")
OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
P = ctypes.c_void_p
A, B_, C, D_, E, F, G, H, I, J = (P(0x100000 * (i + 1)) for i in range(10))   # never dereferenced
INVALID, UNSUPPORTED, WORKSPACE = sb.SOL_ERR_INVALID_ARG, sb.SOL_ERR_UNSUPPORTED, sb.SOL_ERR_WORKSPACE


def strides(*s):
    return (ctypes.c_longlong * len(s))(*s)


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(sol_\w+)\s*\(", text))
    assert names == set(sc.SIGNATURES)
    for name in names:
        assert hasattr(sc.lib(), name), name
    assert re.search(r"SOL_CACHE_PAGE = 64\b", text) and sc.PAGE == 64
    assert re.search(r"SOL_ROPE_HALVES = 0, SOL_ROPE_PAIRS = 1\b", text) and (sc.HALVES, sc.PAIRS) == (0, 1)


def rope(**kw):
    a = dict(q=A, k=B_, qo=C, ko=D_, sq=strides(1, 1, 1), sk=strides(1, 1, 1), sqo=strides(1, 1, 1), sko=strides(1, 1, 1), wq=None,
             wk=None, cos=E, sin=F, pos=G, B=1, Hq=4, Hk=2, N=10, d=128, P=100, rot=128, pairs=0, eps=1e-6, dtype=0, wdtype=0)
    a.update(kw)
    return sc.lib().sol_qk_norm_rope(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), INVALID), (dict(ko=None), INVALID), (dict(Hk=0), INVALID), (dict(qo=A), INVALID), (dict(qo=B_), INVALID),
    (dict(ko=A), INVALID), (dict(ko=C), INVALID), (dict(sq=None), INVALID), (dict(sko=strides(1, -1, 1)), INVALID), (dict(B=0), INVALID),
    (dict(N=-1), INVALID), (dict(d=96), UNSUPPORTED), (dict(dtype=2), INVALID), (dict(wdtype=3), INVALID), (dict(rot=12), INVALID),
    (dict(rot=136), INVALID), (dict(rot=-8), INVALID), (dict(cos=None), INVALID), (dict(P=0), INVALID), (dict(pairs=2), INVALID),
    (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(pos=None, P=9), INVALID),
    (dict(q=None, k=None, qo=None, ko=None, Hq=0, Hk=0), INVALID), (dict(Hq=65535), UNSUPPORTED),
])
def test_rope_refusals(kw, code):
    assert rope(**kw) == code
    assert sb.last_error()


def tables(**kw):
    a = dict(lens=A, add=B_, table=C, ring=D_, state=E, lens_out=F, state_out=G, row_start=H, slots=I, positions=J, S=4, MP=8, P=16,
             rows=5)
    a.update(kw)
    return sc.lib().sol_cache_tables(*a.values(), None)


@pytest.mark.parametrize("kw,code", [(dict([(n, None)]), INVALID) for n in ("lens", "add", "table", "ring", "state", "lens_out",
                                                                          "state_out", "row_start", "slots", "positions")] + [
    (dict(S=0), INVALID), (dict(MP=0), INVALID), (dict(P=0), INVALID), (dict(rows=-1), INVALID), (dict(lens_out=A), INVALID),
    (dict(state_out=E), INVALID), (dict(S=4097), UNSUPPORTED), (dict(P=(1 << 24) + 1), UNSUPPORTED),
    (dict(S=4096, MP=1 << 20), UNSUPPORTED), (dict(rows=(1 << 30) + 1), UNSUPPORTED)])
def test_tables_refusals(kw, code):
    assert tables(**kw) == code
    assert sb.last_error()


def append(**kw):
    a = dict(k=A, v=B_, sk=strides(1, 1), sv=strides(1, 1), store=C, slots=D_, T=4, H=2, d=128, P=4, dtype=0)
    a.update(kw)
    return sc.lib().sol_cache_append(*a.values(), None)


def read(**kw):
    a = dict(store=C, slots=D_, k=A, v=B_, sk=strides(1, 1), sv=strides(1, 1), T=4, H=2, d=128, P=4, dtype=0)
    a.update(kw)
    return sc.lib().sol_cache_read(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), INVALID), (dict(slots=None), INVALID), (dict(store=None), INVALID), (dict(store=P(0x300008)), INVALID),
    (dict(T=0), INVALID), (dict(H=0), INVALID), (dict(P=0), INVALID), (dict(P=1 << 25), UNSUPPORTED), (dict(d=32), UNSUPPORTED),
    (dict(dtype=7), INVALID), (dict(sk=None), INVALID), (dict(sv=strides(1, -2)), INVALID)])
def test_append_and_read_refusals(kw, code):
    assert append(**kw) == code
    if kw == dict(k=None):
        kw = dict(k=None, v=None)
    assert read(**kw) == code
    assert sb.last_error()


def test_too_many_heads():
    for call in (append, read):
        assert call(T=1, H=65536) == UNSUPPORTED
        assert "65,535 heads" in sb.last_error()


def attn(**kw):
    a = dict(q=A, sq=strides(1, 1), out=B_, so=strides(1, 1), store=C, table=D_, lens=E, row_start=F, positions=G, S=2, T=8, rows=4,
             Hq=8, Hk=2, d=128, P=100, MP=50, G=1, dtype=0, ws=H, ws_bytes=1 << 40)
    a.update(kw)
    return sc.lib().sol_cache_forward(*a.values(), None)


@pytest.mark.parametrize("kw,code", [(dict([(n, None)]), INVALID) for n in ("q", "out", "store", "table", "lens", "row_start",
                                                                          "positions", "sq", "so")] + [
    (dict(out=A), INVALID), (dict(store=P(0x300004)), INVALID), (dict(S=0), INVALID), (dict(T=0), INVALID), (dict(rows=0), INVALID),
    (dict(Hq=7), INVALID), (dict(Hk=0), INVALID), (dict(d=80), UNSUPPORTED), (dict(P=0), INVALID), (dict(MP=0), INVALID),
    (dict(G=0), INVALID), (dict(dtype=4), INVALID), (dict(S=4097), UNSUPPORTED), (dict(T=1 << 28), UNSUPPORTED),
    (dict(ws=None), WORKSPACE), (dict(ws_bytes=1000), WORKSPACE), (dict(ws=P(0x800004)), INVALID)])
def test_forward_refusals(kw, code):
    assert attn(**kw) == code
    assert sb.last_error()


def test_sizes():
    assert sc.cache_bytes(10, 3, 128) == 10 * 3 * 68 * 128
    for bad in ((0, 1, 64), (1, 0, 64), (1, 1, 96), (1 << 25, 1, 64)):
        with pytest.raises(ValueError):
            sc.cache_bytes(*bad)
    assert sc.workspace_bytes(4, 4, 1, 8, 2, 128, 1000) > 0
    with pytest.raises(ValueError):
        sc.workspace_bytes(4, 4, 1, 8, 3, 128, 1000)


def test_tensors_are_checked():
    q, k = torch.zeros(1, 4, 6, 64), torch.zeros(1, 2, 6, 64)
    with pytest.raises(ValueError, match="GPU"):
        sc.qk_norm_rope(q, k)
    with pytest.raises(ValueError, match="agree"):
        sc.qk_norm_rope(q, torch.zeros(1, 2, 5, 64))
    with pytest.raises(ValueError, match="contiguous"):
        sc.qk_norm_rope(q.transpose(2, 3), None)
    with pytest.raises(ValueError, match="dtype"):
        sc.qk_norm_rope(q, k.bfloat16())
    with pytest.raises(TypeError):
        sc.qk_norm_rope(q.half(), None)
    with pytest.raises(ValueError, match="overlap"):
        sc.qk_norm_rope(q, None, q_out=q)
    with pytest.raises(ValueError, match="rows of q_out overlap"):
        sc.qk_norm_rope(q, None, q_out=torch.zeros(64).expand(1, 4, 6, 64))
    with pytest.raises(ValueError, match="together"):
        sc.qk_norm_rope(q, k, cos=torch.zeros(6, 32))
    with pytest.raises(ValueError, match="positions"):
        sc.qk_norm_rope(q, k, cos=torch.zeros(6, 32), sin=torch.zeros(6, 32), positions=torch.zeros(6, dtype=torch.int32))
    i32 = dict(dtype=torch.int32)
    lens, add, table, ring, state = torch.zeros(3, **i32), torch.zeros(3, **i32), torch.zeros(3, 4, **i32), torch.zeros(9, **i32), torch.zeros(2, **i32)
    with pytest.raises(ValueError, match="GPU"):
        sc.tables(lens, add, table, ring, state, 5)
    with pytest.raises(ValueError, match="add"):
        sc.tables(lens, add[:2], table, ring, state, 5)
    with pytest.raises(ValueError, match="dtype"):
        sc.tables(lens.long(), add, table, ring, state, 5)
    step = sc.Step(torch.zeros(4, **i32), torch.zeros(5, **i32), torch.zeros(5, **i32), lens, torch.zeros(2, **i32))
    with pytest.raises(ValueError, match="overlap"):
        sc.tables(lens, add, table, ring, state, 5, out=step)
    store = torch.zeros(5, 2, 68 * 64, dtype=torch.uint8)
    k = torch.zeros(2, 7, 64)
    slots = torch.zeros(7, **i32)
    with pytest.raises(ValueError, match="GPU"):
        sc.append(k, k, store, slots)
    with pytest.raises(ValueError, match="heads"):
        sc.append(k[:1], k[:1], store, slots)
    with pytest.raises(ValueError, match="slots"):
        sc.append(k, k, store, slots[:3])
    with pytest.raises(ValueError, match="store"):
        sc.append(k, k, store[:, :, :100], slots)
    with pytest.raises(TypeError):
        sc.read(store, slots, dtype=torch.float16)
    args = (store, table, lens, torch.zeros(4, **i32), torch.zeros(7, **i32))
    q = torch.zeros(4, 7, 64)
    with pytest.raises(ValueError, match="GPU"):
        sc.forward(q, *args)
    with pytest.raises(ValueError, match="channels"):
        sc.forward(torch.zeros(4, 7, 128), *args)
    with pytest.raises(ValueError, match="overlap"):
        sc.forward(q, *args, out=q)
    with pytest.raises(ValueError, match="positions"):
        sc.forward(torch.zeros(4, 8, 64), *args)


def test_reference_quantiser():
    x = np.zeros((1, 32))
    x[0, :10] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 0.2501, -0.25]
    code, e = ora.quantise(x, ora.K_SCALES)
    assert e.tolist() == [[0]]
    assert code[0, :10].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 1, 8]      # ties to the even code
    for top, want in ((7.0, 0), (7.0001, 1), (8.0, 1), (3.99, 0), (3.5, -1), (3.5001, 0), (4.0, 0)):
        assert ora.quantise(np.full((1, 32), top), ora.K_SCALES)[1].tolist() == [[want]], top
    assert ora.quantise(np.full((1, 32), 1e30), ora.V_SCALES)[1].tolist() == [[13]]
    assert ora.quantise(np.full((1, 32), 1e-30), ora.V_SCALES)[1].tolist() == [[-23]]
    assert ora.quantise(np.zeros((1, 32)), ora.K_SCALES)[1].tolist() == [[-100]]


@pytest.mark.parametrize("d", [64, 128])
def test_reference_pages_keep_what_is_written(d):
    rng = np.random.default_rng(d)
    page = np.zeros(68 * d, np.uint8)
    kv = rng.standard_normal((2, 64, d)) * 3
    (kc, ke), (vc, ve) = ora.quantise(kv[0], ora.K_SCALES), ora.quantise(kv[1], ora.V_SCALES)
    for t in rng.permutation(64):
        ora.write_page_token(page, t, d, (kc[t], ke[t]), (vc[t], ve[t]))
    k, v = ora.read_page(page, d)
    assert np.array_equal(k, ora.values(kc, ke)) and np.array_equal(v, ora.values(vc, ve))


def test_reference_tables_by_hand():
    # two requests: 60 tokens on page 3, 64 tokens on page 1; free pages 5, 0 in front
    table = np.array([[3, -1], [1, -1]])
    ring = np.array([5, 0, -1, -1, -1, -1])
    got = ora.tables([60, 64], [6, 1], table, ring, [0, 2], 9)
    assert got[0].tolist() == [0, 6, 7]
    assert got[1].tolist() == [252, 253, 254, 255, 320, 321, 0, -1, -1]
    assert got[2].tolist() == [60, 61, 62, 63, 64, 65, 64, -1, -1]
    assert got[3].tolist() == [66, 65] and got[4].tolist() == [2, 0]
    assert got[5].tolist() == [[3, 5], [1, 0]]
    got = ora.tables(got[3], [-7, 64], got[5], got[6], got[4], 64)      # the first gives page 5 back, the second is refused
    assert got[3].tolist() == [59, 65] and got[4].tolist() == [2, 1] and got[6][2] == 5
    assert (got[1] == -1).all() and (got[2] == -1).all()


def test_sizes_past_a_launch_are_refused():
    assert rope(N=(1 << 27) + 1, P=1 << 28) == UNSUPPORTED
    assert append(T=(1 << 27) + 1) == UNSUPPORTED and read(T=(1 << 27) + 1) == UNSUPPORTED
    assert attn(T=(1 << 21) + 1, rows=1) == UNSUPPORTED
    assert attn(S=4096, T=4096, rows=1, Hq=128, Hk=128) == UNSUPPORTED


def test_device_of_the_tensors_is_made_current_for_the_call(monkeypatch):
    calls = []

    class Guard:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            calls.append(("enter", self.device))

        def __exit__(self, *a):
            calls.append(("exit", self.device))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "device", Guard)
    monkeypatch.setattr(sc, "_stream", lambda device: 100 + device.index)

    def fn(*args):
        calls.append(args)
        return 0
    sc._call(fn, torch.device("cuda", 0), 1, 2)
    assert calls == [(1, 2, 100)]
    calls.clear()
    other = torch.device("cuda", 1)
    sc._call(fn, other, 3)
    assert calls == [("enter", other), (3, 101), ("exit", other)]
    with pytest.raises(sb.SolAttnError):
        sc._call(lambda *a: -1, torch.device("cuda", 0))


def gfx950_objects(path):
    """The gfx950 code objects of a shared library that hipcc linked."""
    data = open(path, "rb").read()
    magic, at, found = b"__CLANG_OFFLOAD_BUNDLE__", 0, []
    while (at := data.find(magic, at)) >= 0:
        entries, = struct.unpack_from("<Q", data, at + len(magic))
        p = at + len(magic) + 8
        for _ in range(entries if entries < 8 else 0):      # the library's own text may hold the word too
            offset, size, n = struct.unpack_from("<QQQ", data, p)
            if b"gfx950" in data[p + 24:p + 24 + n]:
                found.append(data[at + offset:at + offset + size])
            p += 24 + n
        at += len(magic)
    return found


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
def test_conversions_of_queries_keep_results_and_operands_apart(tmp_path):
    """The conversions to and from 6-bit floats write their results before they have read all operands: in no kernel may the two
    share registers."""
    seen = 0
    for i, code in enumerate(gfx950_objects(sb.LIB_PATH)):
        path = tmp_path / f"{i}.o"
        path.write_bytes(code)
        text = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(path)], capture_output=True, text=True, check=True).stdout
        for line in re.findall(r"v_cvt_scalef32_(?:2xpk16_fp6_f32|pk32_f32_fp6)[^/\n]*", text):
            regs = [set(range(int(a), int(b or a) + 1)) for a, b in re.findall(r"\bv\[?(\d+)(?::(\d+))?\]?", line.split(None, 1)[1])]
            assert len(regs) >= 3 and not any(regs[0] & r for r in regs[1:]), line
            seen += 1
    # bf16 rows: three terms and two of them back, f32 six and five, for the blocks of 32 channels of a lane
    assert seen >= 5 * 4 + 11 * 4, seen


@pytest.mark.parametrize("S", [64, 65, 300])
def test_workspace_has_room_for_the_pieces_of_a_plan(S):
    # single tokens, 32 and 8 heads of 128: 12 waves on each of 256 compute units, filled once for up to 64 requests and twice for more, or
    # a piece for each tile where there are more tiles; 64 pieces of slack, 16 rows of 130 floats to a piece
    tiles = (S * 4 // 16 + S) * 8
    pieces = max(tiles, 12 * 256 * (1 if S <= 64 else 2) + 64)
    assert sc.workspace_bytes(S, S, 1, 32, 8, 128, 502) == 256 + pieces * 16 * 130 * 4


def test_workspace_of_tiles_that_no_plan_cuts():
    # 40 heads of a whole 720p video are 23,640 tiles of 128 rows: past 512 workgroups filled seven times they stay whole
    at_most = 512 * 7 + 64
    assert sc.workspace_bytes(1, 75600, 75600, 40, 40, 128, 1200) == 256 + -(-(at_most + 1) // 128) * 128 * 128 * 130 * 4
    assert sc.workspace_bytes(1, 400000, 400000, 40, 40, 128, 7000) == sc.workspace_bytes(1, 75600, 75600, 40, 40, 128, 1200)
    # single tokens of 4,000 requests of 64 heads: 272,000 tiles of 16 rows, the waves filled twice
    assert sc.workspace_bytes(4000, 4000, 1, 64, 64, 64, 502) == 256 + (2 * 12 * 256 + 64) * 16 * 66 * 4


def test_overlap_of_views():
    def cells(t):
        at = torch.zeros((), dtype=torch.long)
        for st, n in zip(t.stride(), t.shape):
            at = at[..., None] + torch.arange(n) * st
        return set(((t.data_ptr() + (at * t.element_size()).flatten()[:, None] + torch.arange(t.element_size())).flatten()).tolist())
    rng = np.random.default_rng(0)
    buffer = torch.zeros(4000)
    apart = 0
    for _ in range(3000):
        views = []
        for _ in range(2):
            unit, rows = int(rng.choice([24, 48, 72])), int(rng.integers(1, 9))
            heads, width = int(rng.integers(1, 4)), int(rng.integers(1, 9))
            views.append(buffer.as_strided((rows, heads, width), (unit, int(rng.choice([8, 12])), 1), int(rng.integers(0, 100))))
        if rng.random() < 0.3:
            views[1] = views[1].view(torch.int32) if rng.random() < 0.5 else views[1].transpose(0, 1)
        shared = bool(cells(views[0]) & cells(views[1]))
        assert sc._overlap(*views) or not shared
        apart += not sc._overlap(*views) and views[0].data_ptr() < views[1].data_ptr() + 4 * 24
    assert apart > 100


def test_outputs_may_lie_in_one_buffer():
    """Parts of the rows of one buffer, as a projection's output has them: no output shares memory with another tensor."""
    rows = torch.zeros(2, 10, 16, 64)                            # [B, N, 8 heads of q, 4 of k, 4 that are free, 64]
    q, k, free = (rows[:, :, a:b].transpose(1, 2) for a, b in ((0, 8), (8, 12), (12, 16)))
    other = torch.zeros(2, 10, 12, 64)
    q_out, k_out = other[:, :, :8].transpose(1, 2), other[:, :, 8:].transpose(1, 2)
    for call in (lambda: sc.qk_norm_rope(q, k, q_out=q_out, k_out=k_out), lambda: sc.qk_norm_rope(None, k, k_out=free)):
        with pytest.raises(ValueError, match="GPU"):             # nothing else is wrong
            call()
    for call in (lambda: sc.qk_norm_rope(q, k, k_out=q[:, 4:]), lambda: sc.qk_norm_rope(q, k, q_out=q_out, k_out=q_out[:, 1:5])):
        with pytest.raises(ValueError, match="overlap"):
            call()
    store, slots = torch.zeros(3, 4, 68 * 64, dtype=torch.uint8), torch.zeros(10, dtype=torch.int32)
    kv = torch.zeros(10, 2, 4, 64).transpose(0, 2)               # [4, 2, 10, 64]
    with pytest.raises(ValueError, match="GPU"):
        sc.read(store, slots, k_out=kv[:, 0], v_out=kv[:, 1])
    with pytest.raises(ValueError, match="overlap"):
        sc.read(store, slots, k_out=kv[:, 0], v_out=kv[:, 0])
    i32 = dict(dtype=torch.int32)
    args = (store, torch.zeros(1, 2, **i32), torch.zeros(1, **i32), torch.zeros(2, **i32), torch.zeros(10, **i32))
    with pytest.raises(ValueError, match="GPU"):
        sc.forward(q[0], *args, out=torch.zeros(10, 16, 64)[:, :8].transpose(0, 1))
    with pytest.raises(ValueError, match="GPU"):
        sc.forward(q[0, :4], *args, out=free[0])
    with pytest.raises(ValueError, match="overlap"):
        sc.forward(q[0], *args, out=rows[0, :, 2:10].transpose(0, 1))


@pytest.mark.parametrize("size,want", [(1.0, 0.159), (2.0, 0.251)])
def test_error_that_the_cache_brings(size, want):
    """Attention over what the cache holds against attention on the keys and values themselves, normal data.

    Keys and values are each off by 11.2 % of theirs.  With queries of the root mean square `size` a logit has that standard deviation, and
    an error of 0.112 times it; an output, a sum over many keys, is off by the root of that squared and 0.112 squared.  2,048
    values that share their weights by 128: within an eighth."""
    rng = np.random.default_rng(3)
    L, d, rows = 4096, 128, 16
    k, v = rng.standard_normal((2, L, d))
    q = size * rng.standard_normal((rows, d))
    held = [ora.values(*ora.quantise(x, limits)) for x, limits in ((k, ora.K_SCALES), (v, ora.V_SCALES))]
    for x, y in zip((k, v), held):
        assert abs(np.linalg.norm(x - y) / np.linalg.norm(x) - 0.112) < 0.001
    sees = np.ones((rows, L), bool)
    a, b = ora.attend(q, k, v, sees)[0], ora.attend(q, *held, sees)[0]
    off = np.linalg.norm(a - b) / np.linalg.norm(a)
    assert abs(off - want) < want / 8, off
