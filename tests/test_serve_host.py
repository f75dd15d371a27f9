"""The operators beside the products without a GPU: what they refuse, what their structures look like, their references."""
import ctypes as C
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

from paper_2605_11582_amd import binding as egt
import serve_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                # a made-up address: nothing follows it on the host
NULL, SHAPE, BUFFER, UNSUPPORTED = 1, 2, 5, 6
MIRRORS = {"egt_kv_cache": egt.KvCache, "egt_slots_batch": egt.SlotsBatch, "egt_append_batch": egt.AppendBatch, "egt_tree_batch": egt.TreeBatch,
           "egt_lora_batch": egt.LoraBatch, "egt_rules_batch": egt.RulesBatch}


def test_structures_are_those_of_the_header(tmp_path):
    cc = shutil.which("gcc")
    if not cc:
        pytest.skip("no host compiler")
    lines = []
    for name, mirror in MIRRORS.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f}));' for f, _ in mirror._fields_]
    (tmp_path / "s.c").write_text('#include <stdio.h>\n#include "egt.h"\nint main(void) {' + "\n".join(lines) + "return 0; }\n")
    subprocess.run([cc, "-I" + os.path.join(ROOT, "include"), str(tmp_path / "s.c"), "-o", str(tmp_path / "s")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for mirror in MIRRORS.values():
        want += [C.sizeof(mirror)] + [getattr(mirror, f).offset for f, _ in mirror._fields_]
    assert got == want


def cache(**change):
    c = dict(k=P, v=P, blocks=8, heads=2, page=16, dim=64, k_block=2048, k_head=1024, k_token=64, v_block=2048, v_head=1024, v_token=64)
    return egt.KvCache(**{**c, **change})


def slots(**change):
    b = dict(lens=P, counts=P, block_table=P, free_blocks=P, free_head=P, slots=P, cu_tokens=P, new_lens=2 * P, new_head=2 * P, ld_table=4, requests=3,
             table_blocks=4, page=16, blocks=8, n_free=5, n_slots=7)
    return egt.SlotsBatch(**{**b, **change})


def append(**change):
    return egt.AppendBatch(**{**dict(k=P, v=P, slots=P, k_row=128, k_head=64, v_row=128, v_head=64, n=4, n_rows=4), **change})


def tree(**change):
    b = dict(q=P, k=P, v=P, out=P, q_row=256, q_head=64, k_row=128, k_head=64, v_row=128, v_head=64, out_row=256, out_head=64, block_table=P, lens=P,
             cu_tokens=P, mask=P, ld_table=4, requests=3, tokens=9, heads=4, max_tokens=5, table_blocks=4, scale=0.125)
    return egt.TreeBatch(**{**b, **change})


def lora(**change):
    b = dict(X=P, A=P, B=P, base=P, Y=P, index=P, scale=P, ldx=64, ldbase=100, ldy=100, a_stride=512, b_stride=800, M=4, cols=64, rows=100, rank=8, adapters=3)
    return egt.LoraBatch(**{**b, **change})


def rules(**change):
    b = dict(logits=P, out=P, cu_tokens=P, history=P, history_len=P, draft=P, mask=P, bias_ids=P, bias=P, allowed=P, allowed_row=P, ld_logits=100,
             ld_out=100, ld_history=10, ld_allowed=4, kind=0, requests=2, tokens=5, vocab=100, history_width=10, n_bias=3, n_allowed=2)
    return egt.RulesBatch(**{**b, **change})


@pytest.mark.parametrize("change,status", [
    (dict(requests=0), SHAPE), (dict(requests=egt.MAX_REQUESTS + 1), UNSUPPORTED), (dict(page=12), SHAPE), (dict(page=0), SHAPE), (dict(ld_table=3), SHAPE),
    (dict(table_blocks=-1), SHAPE), (dict(n_slots=-1), SHAPE), (dict(n_free=-1), SHAPE), (dict(blocks=1 << 27), SHAPE), (dict(lens=None), NULL),
    (dict(counts=None), NULL), (dict(block_table=None), NULL), (dict(free_blocks=None), NULL), (dict(free_head=None), NULL), (dict(slots=None), NULL),
    (dict(cu_tokens=None), NULL), (dict(new_lens=None), NULL), (dict(new_head=None), NULL), (dict(new_lens=P), BUFFER), (dict(new_head=P), BUFFER),
    (dict(slots=P + 2), BUFFER), (dict(lens=P + 1), BUFFER)])
def test_kv_slots_refuses(change, status):
    assert egt.lib().egt_kv_slots(C.byref(slots(**change)), None) == status


@pytest.mark.parametrize("change,cached,status", [
    (dict(n=-1), {}, SHAPE), (dict(n_rows=-1), {}, SHAPE), (dict(k=None), {}, NULL), (dict(v=None), {}, NULL), (dict(slots=None), {}, NULL), (dict(k=P + 8), {}, BUFFER),
    (dict(k_row=4), {}, BUFFER), (dict(v_head=-64), {}, BUFFER), (dict(slots=P + 2), {}, BUFFER), ({}, dict(page=6), SHAPE), ({}, dict(dim=12), SHAPE),
    ({}, dict(dim=264), SHAPE), ({}, dict(heads=0), SHAPE), ({}, dict(blocks=-1), SHAPE), ({}, dict(blocks=1 << 27), SHAPE), ({}, dict(k=None), NULL),
    ({}, dict(v=None), NULL), ({}, dict(k_token=68), BUFFER), ({}, dict(v=P + 2), BUFFER), ({}, dict(v_block=-2048), BUFFER),
    (dict(n=0, k=None), {}, 0), (dict(n_rows=0, k=None), {}, 0), (dict(k=None), dict(blocks=0, k=None, v=None), 0)])
def test_kv_append_refuses(change, cached, status):
    assert egt.lib().egt_kv_append(C.byref(append(**change)), C.byref(cache(**cached)), None) == status


@pytest.mark.parametrize("change,cached,status", [
    (dict(heads=3), {}, SHAPE), (dict(heads=0), {}, SHAPE), (dict(max_tokens=0), {}, SHAPE), (dict(max_tokens=65), {}, SHAPE), (dict(requests=-1), {}, SHAPE),
    (dict(tokens=-1), {}, SHAPE), (dict(table_blocks=-1), {}, SHAPE), (dict(ld_table=3), {}, SHAPE), (dict(scale=float("nan")), {}, SHAPE),
    (dict(table_blocks=1 << 28, ld_table=1 << 28), {}, SHAPE), (dict(requests=egt.MAX_REQUESTS + 1), {}, UNSUPPORTED), ({}, dict(dim=20), SHAPE),
    ({}, dict(page=24), SHAPE), (dict(q=None), {}, NULL), (dict(k=None), {}, NULL), (dict(v=None), {}, NULL), (dict(out=None), {}, NULL), (dict(lens=None), {}, NULL),
    (dict(cu_tokens=None), {}, NULL), (dict(mask=None), {}, NULL), (dict(block_table=None), {}, NULL), (dict(q=P + 8), {}, BUFFER), (dict(out=P + 4), {}, BUFFER),
    (dict(q_row=260), {}, BUFFER), (dict(out_head=60), {}, BUFFER), (dict(mask=P + 4), {}, BUFFER), (dict(lens=P + 2), {}, BUFFER), ({}, dict(k_token=60), BUFFER),
    (dict(requests=0, q=None), {}, 0), (dict(tokens=0, q=None), {}, 0)])
def test_tree_attention_refuses(change, cached, status):
    L, b, c = egt.lib(), tree(**change), cache(**cached)
    assert L.egt_tree_attention(C.byref(b), C.byref(c), P, 1 << 30, None) == status


def test_tree_attention_workspace():
    L, n = egt.lib(), C.c_size_t()
    for change in ({}, dict(max_tokens=64, heads=64), dict(table_blocks=1 << 20, requests=1), dict(requests=64, table_blocks=4096)):
        b, c = tree(**{**change, "q": None, "k": None, "out": None}), cache(k=None, v=None)
        assert L.egt_tree_attention_ws_bytes(C.byref(b), C.byref(c), C.byref(n)) == 0 and n.value >= 16 and n.value % 16 == 0
        b, c, need = tree(**{**change, "ld_table": 1 << 20}), cache(), n.value
        assert L.egt_tree_attention(C.byref(b), C.byref(c), None, need, None) == NULL
        assert L.egt_tree_attention(C.byref(b), C.byref(c), P, need - 1, None) == SHAPE
        assert L.egt_tree_attention(C.byref(b), C.byref(c), P + 8, need, None) == BUFFER
    assert L.egt_tree_attention_ws_bytes(C.byref(tree()), C.byref(cache()), None) == NULL
    assert L.egt_tree_attention_ws_bytes(C.byref(tree(max_tokens=65)), C.byref(cache()), C.byref(n)) == SHAPE


@pytest.mark.parametrize("change,status", [
    (dict(M=0), SHAPE), (dict(M=65), SHAPE), (dict(cols=60), SHAPE), (dict(rank=12), SHAPE), (dict(rank=0), SHAPE), (dict(rank=136), UNSUPPORTED),
    (dict(rows=-1), SHAPE), (dict(adapters=0), SHAPE), (dict(ldx=56), SHAPE), (dict(ldy=99), SHAPE), (dict(ldbase=99), SHAPE), (dict(ldbase=104), SHAPE),
    (dict(a_stride=-8), SHAPE), (dict(X=None), NULL), (dict(A=None), NULL), (dict(B=None), NULL), (dict(Y=None), NULL), (dict(index=None), NULL),
    (dict(X=P + 8), BUFFER), (dict(A=P + 2), BUFFER), (dict(ldx=68), BUFFER), (dict(b_stride=804), BUFFER), (dict(index=P + 1), BUFFER), (dict(rows=0, X=None), 0)])
def test_lora_smallm_refuses(change, status):
    b = lora(**change)
    assert egt.lib().egt_lora_smallm(C.byref(b), P, 1 << 30, None) == status


def test_lora_smallm_workspace():
    L, n = egt.lib(), C.c_size_t()
    for M, cols, rank in ((1, 8, 8), (64, 4096, 16), (64, 16384, 128)):
        assert L.egt_lora_smallm_ws_bytes(M, cols, rank, C.byref(n)) == 0 and n.value >= 16
        b = lora(M=M, cols=cols, ldx=cols, rank=rank)
        assert L.egt_lora_smallm(C.byref(b), P, n.value - 1, None) == SHAPE
        assert L.egt_lora_smallm(C.byref(b), None, n.value, None) == NULL
    assert L.egt_lora_smallm_ws_bytes(65, 8, 8, C.byref(n)) == SHAPE and L.egt_lora_smallm_ws_bytes(1, 8, 8, None) == NULL


@pytest.mark.parametrize("change,status", [
    (dict(kind=2), SHAPE), (dict(requests=-1), SHAPE), (dict(tokens=-1), SHAPE), (dict(vocab=-1), SHAPE), (dict(ld_logits=99), SHAPE), (dict(ld_out=99), SHAPE),
    (dict(ld_out=104), SHAPE), (dict(ld_history=9), SHAPE), (dict(history_width=-1), SHAPE), (dict(ld_allowed=3), SHAPE), (dict(n_bias=-1), SHAPE),
    (dict(requests=egt.MAX_REQUESTS + 1), UNSUPPORTED), (dict(logits=None), NULL), (dict(out=None), NULL), (dict(cu_tokens=None), NULL), (dict(history_len=None), NULL),
    (dict(mask=None), NULL), (dict(bias=None), NULL), (dict(allowed_row=None), NULL), (dict(logits=P + 1, out=2 * P), BUFFER), (dict(kind=1, out=2 * P + 2), BUFFER),
    (dict(mask=P + 4), BUFFER), (dict(history=P + 2), BUFFER), (dict(requests=0, logits=None), 0), (dict(tokens=0, logits=None), 0), (dict(vocab=0, logits=None), 0)])
def test_logits_rules_refuses(change, status):
    assert egt.lib().egt_logits_rules(C.byref(rules(**change)), None) == status


def test_rows_of_a_grammar_need_a_grammar():
    """An empty grammar's missing address is not "everything is allowed"."""
    assert egt.lib().egt_logits_rules(C.byref(rules(allowed=None, n_allowed=0)), None) == NULL
    assert egt.lib().egt_logits_rules(C.byref(rules(allowed=None, allowed_row=None, n_allowed=0, cu_tokens=P + 2)), None) == BUFFER      # (neither: as ever)


def test_the_binding_names_what_is_wrong():
    i, h = torch.zeros(4, dtype=torch.int32), torch.zeros((4, 2, 8), dtype=torch.float16)
    with pytest.raises(ValueError, match="lens: expected a device tensor"):
        egt.kv_slots(i, i, i.view(4, 1), 16, 4, i, i[:1], i, i, i, i[:1])
    with pytest.raises(ValueError, match="k: expected a device tensor"):
        egt.kv_append(h, h, i, h, h)
    with pytest.raises(ValueError, match="q: expected a device tensor"):
        egt.tree_attention(h, h, h, h, h, i, i, i, i, h, 1.0)
    with pytest.raises(ValueError, match="X: expected a device tensor"):
        egt.lora_smallm(h[0], h, h, i, h[0], None)
    with pytest.raises(ValueError, match="logits: expected a device tensor"):
        egt.logits_rules(h[0], h[0], i)
    with pytest.raises(ValueError, match="logits"):
        egt.prepared_logits_rules(None, h[0], i)
    with pytest.raises(TypeError):
        egt._native().kv_slots(False, i)


def test_tensors_without_memory_are_refused():
    from torch._subclasses.fake_tensor import FakeTensorMode

    def body(t, i):
        for call in (lambda: egt.kv_append(t, t, i, t[None], t[None]), lambda: egt.logits_rules(t[0], t[0], i), lambda: egt.prepared_logits_rules(t[0], t[0], i)):
            with pytest.raises(ValueError):
                call()
        return t
    with FakeTensorMode():
        torch.vmap(body)(torch.empty((3, 4, 8, 64), dtype=torch.float16, device="cuda"), torch.empty((3, 4), dtype=torch.int32, device="cuda"))


LAUNCHES = r"""
import ctypes as C, itertools, sys
sys.path.insert(0, {root!r})
sys.path.insert(0, {root!r} + "/tests")
from paper_2605_11582_amd import binding as B
L, P = B._declare(C.CDLL(B.LIB_PATH)), 1 << 20             # (without PyTorch)
need = C.c_size_t()
for dim, kv, group, most, requests, table, page in itertools.product((8, 64, 72, 96, 128, 160, 192, 200, 256), (1, 8), (1, 3, 16), (1, 7, 64), (1, 40, 8192), (0, 3, 4096), (1, 16)):
    heads = kv * group
    c = B.KvCache(k=P, v=P, blocks=8, heads=kv, page=page, dim=dim, k_block=8, k_head=8, k_token=8, v_block=8, v_head=8, v_token=8)
    b = B.TreeBatch(q=P, k=P, v=P, out=P, q_row=8, q_head=8, k_row=8, k_head=8, v_row=8, v_head=8, out_row=8, out_head=8, block_table=P, lens=P, cu_tokens=P, mask=P,
                    ld_table=table, requests=requests, tokens=requests * most, heads=heads, max_tokens=most, table_blocks=table, scale=1.0)
    assert L.egt_tree_attention_ws_bytes(C.byref(b), C.byref(c), C.byref(need)) == 0
    print("case", dim, kv, group, most, requests, table, page, need.value, flush=True)
    assert L.egt_tree_attention(C.byref(b), C.byref(c), P, need.value, None) == 0
"""


def test_launches_of_tree_attention(tmp_path):
    """Every shape has a kernel, with LDS that a compute unit has, a grid that the runtime takes, and partial results that fit the workspace
    (a stand-in for the runtime's launch writes down what would run)."""
    import test_kernel_routes as routes
    cc = shutil.which("gcc")
    if not cc:
        pytest.skip("no host compiler")
    lib = str(tmp_path / "launch.so")
    (tmp_path / "launch.c").write_text(routes.STAND_IN.replace('printf("launch %s %u %u %u %zu\\n", name, grid.x, grid.y, block.x, lds);',
                                                               'printf("launch %s %u %u %u %u %zu\\n", name, grid.x, grid.y, grid.z, block.x, lds);'))
    subprocess.run([cc, "-shared", "-fPIC", "-O1", str(tmp_path / "launch.c"), "-o", lib], check=True)
    env = dict(os.environ)
    env["LD_PRELOAD"] = " ".join(v for v in (lib, env.get("LD_PRELOAD", "")) if v)
    out = subprocess.run([os.sys.executable, "-c", LAUNCHES.replace("{root!r}", repr(ROOT))], capture_output=True, text=True, env=env, timeout=300)
    assert out.returncode == 0, (out.stdout[-300:], out.stderr[-2000:])
    case, kernels = None, set()
    for line in out.stdout.splitlines():
        word = line.split()
        if word[0] == "case":
            dim, kv, group, most, requests, table, page, need = (int(w) for w in word[1:])
            case, launches = line, []
            continue
        x, y, z, threads, lds = (int(w) for w in word[2:])
        launches.append(word[1])
        assert 1 <= x and 1 <= y <= 65535 and 1 <= z <= 65535 and x * threads < 1 << 32 and threads <= 1024 and lds <= 158 * 1024, (case, line)
        if "k_tree_join" in word[1]:
            splits = first[0]
            assert len(launches) == 2 and 1 < splits <= 64 and need >= 4 * splits * requests * most * kv * group * (dim + 2), (case, line)
        else:
            first = (x, y, z)
            kernels.add(word[1])
            assert len(launches) == 1 and z == requests and y % kv == 0, (case, line)
    assert len(kernels) >= 20


OTHER_LAUNCHES = r"""
import ctypes as C, sys
sys.path.insert(0, {root!r})
from paper_2605_11582_amd import binding as B
L, P = B._declare(C.CDLL(B.LIB_PATH)), 1 << 20             # (without PyTorch)
for requests in (1, 3, 64, 65, 1000, 8192):
    print("case slots", requests, flush=True)
    b = B.SlotsBatch(lens=P, counts=P, block_table=P, free_blocks=P, free_head=P, slots=P, cu_tokens=P, new_lens=2 * P, new_head=2 * P, ld_table=4, requests=requests,
                     table_blocks=4, page=16, blocks=8, n_free=5, n_slots=7)
    assert L.egt_kv_slots(C.byref(b), None) == 0
for rows, ld in ((1, 1), (64, 64), (2100, 2100), (4100, 4101), (11008, 11008), (65536, 65536), ((1 << 30) - 64, (1 << 30) - 64), ((1 << 30) - 64, (1 << 30) - 63),
                 ((1 << 30) - 63, (1 << 30) - 63), (1 << 30, 1 << 30)):
    for M, rank in ((1, 8), (64, 32), (64, 64), (64, 128)):
        b = B.LoraBatch(X=P, A=P, B=P, base=P, Y=P, index=P, scale=P, ldx=64, ldbase=ld, ldy=ld, a_stride=512, b_stride=800, M=M, cols=64, rows=rows, rank=rank, adapters=M)
        print("case lora", rows, M, rank, flush=True)
        print("status", L.egt_lora_smallm(C.byref(b), P, 1 << 30, None), flush=True)
for heads, dim, n in ((1, 8, 1), (8, 128, (1 << 24) - 1), (1 << 20, 256, 5), (1 << 25, 256, 5), (1 << 26, 256, 5), ((1 << 31) - 1, 8, 5), ((1 << 31) - 1, 256, 5)):
    c = B.KvCache(k=P, v=P, blocks=8, heads=heads, page=16, dim=dim, k_block=2048, k_head=1024, k_token=64, v_block=2048, v_head=1024, v_token=64)
    b = B.AppendBatch(k=P, v=P, slots=P, k_row=128, k_head=64, v_row=128, v_head=64, n=n, n_rows=n)
    print("case append", heads, dim, flush=True)
    print("status", L.egt_kv_append(C.byref(b), C.byref(c), None), flush=True)
for dim, kv, group, tokens, context in {forms!r}:
    for page in (1, 16, 64):
        table = -(-context // page) + 1
        c = B.KvCache(k=P, v=P, blocks=8, heads=kv, page=page, dim=dim, k_block=8, k_head=8, k_token=8, v_block=8, v_head=8, v_token=8)
        b = B.TreeBatch(q=P, k=P, v=P, out=P, q_row=8, q_head=8, k_row=8, k_head=8, v_row=8, v_head=8, out_row=8, out_head=8, block_table=P, lens=P, cu_tokens=P, mask=P,
                        ld_table=table, requests=3, tokens=3 * tokens, heads=kv * group, max_tokens=tokens, table_blocks=table, scale=1.0)
        print("case form", dim, context, flush=True)
        print("status", L.egt_tree_attention(C.byref(b), C.byref(c), P, 1 << 40, None), flush=True)
for rows, rank, pad in {adapters!r}:
    b = B.LoraBatch(X=P, A=P, B=P, base=P, Y=P, index=P, scale=P, ldx=72, ldbase=rows + pad, ldy=rows + pad, a_stride=512, b_stride=800, M=64, cols=72, rows=rows, rank=rank, adapters=64)
    print("case adapter", rows, rank, flush=True)
    print("status", L.egt_lora_smallm(C.byref(b), P, 1 << 30, None), flush=True)
"""


@pytest.fixture(scope="module")
def other_launches(tmp_path_factory):
    """[(case, [(kernel, grid x, grid y, threads, LDS bytes)])]: what runs of the calls above, as a stand-in for the runtime's launch sees it."""
    import test_gpu_serve as on_the_gpu
    import test_kernel_routes as routes
    cc = shutil.which("gcc")
    if not cc:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("launch")
    (d / "launch.c").write_text(routes.STAND_IN)
    subprocess.run([cc, "-shared", "-fPIC", "-O1", str(d / "launch.c"), "-o", str(d / "launch.so")], check=True)
    env = {**os.environ, "LD_PRELOAD": " ".join(v for v in (str(d / "launch.so"), os.environ.get("LD_PRELOAD", "")) if v)}
    script = OTHER_LAUNCHES.replace("{root!r}", repr(ROOT)).replace("{forms!r}", repr(on_the_gpu.FORMS)).replace("{adapters!r}", repr(on_the_gpu.ADAPTER_FORMS))
    out = subprocess.run([os.sys.executable, "-c", script], capture_output=True, text=True, env=env, timeout=120)
    assert out.returncode == 0, (out.stdout[-300:], out.stderr[-2000:])
    seen = []
    for line in out.stdout.splitlines():
        word = line.split()
        if word[0] == "case":
            seen.append((word[1:], []))
        elif word[0] == "status":
            seen[-1] = (seen[-1][0] + [int(word[1])], seen[-1][1])
        else:
            seen[-1][1].append((word[1], *(int(w) for w in word[2:])))
    return seen


def test_waves_of_the_slot_maps_have_lds_of_their_own(other_launches):
    """Up to 64 requests every wave keeps offsets, pages and lengths for itself; beyond, the workgroup shares offsets and pages."""
    for (_, requests), [(name, _, _, threads, lds)] in (c for c in other_launches if c[0][0] == "slots"):
        n = int(requests)
        assert lds == 4 * (threads // 64 * (3 * n + 1) if n <= 64 else 2 * n + 1), (requests, name)


def test_launches_of_adapters_and_cache_writes(other_launches):
    """A grid that a launch takes (less than 2^32 threads), or EGT_ERR_UNSUPPORTED and no launch; a token's pieces are counted in 31 bits."""
    kernels = set()
    for (what, *sizes, status), launches in (c for c in other_launches if c[0][0] in ("lora", "append")):
        sizes = [int(v) for v in sizes]
        fits = sizes[0] <= (1 << 30) - 64 if what == "lora" else sizes[0] * (sizes[1] // 8) <= 1 << 30
        assert status == (0 if fits else UNSUPPORTED) and len(launches) == ((2 if what == "lora" else 1) if fits else 0), (what, sizes)
        for name, x, y, threads, lds in launches:
            assert x * threads < 1 << 32 and y <= 65535, (what, sizes, name)
            kernels.add(name)
    assert len([k for k in kernels if "k_lora_expand" in k]) == 11


def test_the_gpu_tests_reach_every_kernel(other_launches):
    """What the library launches for the cases of the tests on the GPU: every form of the attention, in one span and in several, and
    every form of the adapters' second product."""
    def names(launches):
        text = subprocess.run(["c++filt"], input="\n".join(l[0] for l in launches), capture_output=True, text=True).stdout
        return set(re.findall(r"k_\w+<[^>]*>|k_tree_join", text))
    one, several, adapters = set(), set(), set()
    for (what, *rest), launches in other_launches:
        if what in ("form", "adapter"):
            assert rest[-1] == 0
            found = names(launches)
            if what == "adapter":
                adapters |= {k for k in found if "expand" in k}
            else:
                (several if "k_tree_join" in found else one).update(k for k in found if k != "k_tree_join")
    assert len(one) == len(several) == 23 and one == several and len(adapters) == 11


BIG = 1 << 30


@pytest.mark.parametrize("status,call", [
    (UNSUPPORTED, lambda L: L.egt_kv_append(C.byref(append(n=1 << 24)), C.byref(cache()), None)),
    (SHAPE, lambda L: L.egt_tree_attention(C.byref(tree(scale=float("inf"))), C.byref(cache()), P, BIG, None)),
    (SHAPE, lambda L: L.egt_tree_attention(C.byref(tree(scale=-2.0 ** 127)), C.byref(cache()), P, BIG, None)),
    (UNSUPPORTED, lambda L: L.egt_lora_smallm(C.byref(lora(rows=BIG + 1, ldy=BIG + 1, ldbase=BIG + 1)), P, BIG, None)),
    (UNSUPPORTED, lambda L: L.egt_lora_smallm(C.byref(lora(cols=BIG + 8, ldx=BIG + 8)), P, BIG, None)),
    (UNSUPPORTED, lambda L: L.egt_logits_rules(C.byref(rules(history_width=(1 << 29) + 1, ld_history=BIG)), None)),
    (UNSUPPORTED, lambda L: L.egt_logits_rules(C.byref(rules(n_bias=(1 << 29) + 1)), None))])
def test_sizes_past_what_a_kernel_counts(status, call):
    assert call(egt.lib()) == status


# ---------------------------------------------------------------- the references themselves, on numbers worked out by hand
def test_reference_of_slots():
    lens, counts = np.array([3, 0, 4]), np.array([2, 1, 4])
    table = np.array([[7, -1], [-1, -1], [5, -1]], dtype=np.int32)
    slots_, cu, new, head, table = R.kv_slots(lens, counts, table, 4, 10, np.array([9, 2, 3, 4]), 1, 8)
    # request 0 fills place 3 of page 7, then takes page 2; request 1 takes 3; request 2, whose page is full, takes 4
    assert slots_.tolist() == [31, 8, 12, 16, 17, 18, 19, -1] and cu.tolist() == [0, 2, 3, 7] and new.tolist() == [5, 1, 8] and head.tolist() == [4]
    assert table.tolist() == [[7, 2], [3, -1], [5, 4]]
    slots_, _, new, head, _ = R.kv_slots(lens, counts, np.array([[7, -1], [-1, -1], [5, -1]], dtype=np.int32), 4, 10, np.array([9, 2]), 1, 8)
    assert slots_.tolist() == [31, 8, -1, -1, -1, -1, -1, -1] and new.tolist() == [5, 0, 4] and head.tolist() == [2]


def test_reference_of_attention():
    q = np.array([[[1.0, 0.0]], [[0.0, 1.0]]])
    k = np.array([[[0.0, 0.0]], [[0.0, np.log(3.0)]]])
    v = np.array([[[1.0, 2.0]], [[5.0, 6.0]]])
    kc = np.array([[[[np.log(2.0), 0.0]]]])
    vc = np.array([[[[4.0, 8.0]]]])
    out, _ = R.tree_attention(q, k, v, kc, vc, np.array([[0]]), np.array([1]), [0, 2], np.array([1, 2], np.uint64), 1.0)
    # token 0: weights 2 (cached) and 1 (itself); token 1: weights 1 (cached) and 3 (itself)
    assert np.allclose(out[0, 0], [3.0, 6.0]) and np.allclose(out[1, 0], [(4 + 15) / 4, (8 + 18) / 4])
    out, _ = R.tree_attention(q, k, v, kc, vc, np.array([[0]]), np.array([0]), [0, 2], np.array([0, 1], np.uint64), 1.0)
    assert np.all(out[0] == 0) and np.allclose(out[1, 0], [1.0, 2.0])


def test_reference_of_rules():
    x = np.array([[2.0, -2.0, 1.0, 4.0, 0.5]])
    out, _ = R.rules(x, [0, 1], False, history=np.array([[1, 0, 0, 9, 2]]), history_len=np.array([4]), prompt_len=np.array([1]), draft=np.array([3]),
                     mask=np.array([1], np.uint64), repetition=np.array([2.0]), frequency=np.array([0.25]), presence=np.array([0.5]),
                     bias_ids=np.array([[4, 3, 4]]), bias=np.array([[1.0, -1.0, 3.0]]), allowed=np.array([[0b11011]], np.int32), allowed_row=np.array([0]))
    assert out.tolist() == [[2 / 2 - 0.5 - 0.5, -4.0, -np.inf, 4 / 2 - 0.25 - 0.5 - 1, 3.5]]
