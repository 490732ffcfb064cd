"""Operators for sampled and drafted tokens: what the host decides -- refusals of the C ABI and of the binding, argument
structures, frequencies for long contexts.  No GPU."""
import ctypes as C
import math
import os
import subprocess
import tempfile

import pytest
import torch

from paper_2608_12385_b200 import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PTR = 0x10000  # an aligned address that a refused call does not touch


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


STRUCTS = {
    "dbt_sampling": (binding.SAMPLING_FORMAT, "reserved uniforms temperature top_k top_p min_p"),
    "dbt_rope_spec": (binding.ROPE_SPEC_FORMAT, "kind rot_dim reserved base factor trained_len low high"),
    "dbt_rope_append_args": (binding.ROPE_APPEND_FORMAT,
                             "dtype B max_nodes n_q_heads n_kv_heads head_dim rot_dim interleaved num_pages pages_per_seq scale q k v q_stride[0] "
                             "q_stride[1] q_stride[2] k_stride[0] k_stride[1] k_stride[2] v_stride[0] v_stride[1] v_stride[2] q_out cache_layer "
                             "positions page_table seq_lens node_counts freq status_dev"),
    "dbt_attn_tree_args": (binding.ATTN_TREE_FORMAT,
                           "dtype B max_nodes n_q_heads n_kv_heads head_dim num_pages pages_per_seq softmax_scale q cache_layer q_stride[0] q_stride[1] "
                           "q_stride[2] out page_table seq_lens node_counts parents workspace workspace_bytes status_dev"),
    "dbt_tree_accept_args": (binding.TREE_ACCEPT_FORMAT,
                             "dtype B max_nodes n_layers n_kv_heads head_dim num_pages pages_per_seq tokens parents sampled page_table seq_lens "
                             "node_counts pool path counts next_tokens new_lens status_dev"),
}


@pytest.mark.parametrize("name", sorted(STRUCTS))
def test_argument_formats_have_the_headers_layout(name):
    """A structure packed by the binding, read field by field by the C compiler's layout."""
    fmt, fields = STRUCTS[name]
    fields = fields.split()
    n = len(fields) + 1
    packed = fmt.pack(*range(1, n + 1))
    lines = ['#include "dbt.h"', "#include <stdio.h>", "#include <string.h>", "int main(void) {", f"{name} a;", f"unsigned char raw[{fmt.size}];",
             f'if (fread(raw, 1, {fmt.size}, stdin) != {fmt.size} || sizeof a != {fmt.size}) return 1;', "memcpy(&a, raw, sizeof a);",
             'printf("%.0f ", (double)a.struct_size);']
    lines += [f'printf("%.0f ", (double)({"(size_t)" if fmt.format.count("P") and f.split("[")[0] in POINTERS else ""}a.{f}));' for f in fields]
    lines += ["return 0; }"]
    with tempfile.TemporaryDirectory() as td:
        src, exe = os.path.join(td, "a.c"), os.path.join(td, "a")
        open(src, "w").write("\n".join(lines))
        subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", exe, src], check=True)
        out = subprocess.run([exe], input=packed, check=True, capture_output=True).stdout
    assert [int(x) for x in out.split()] == list(range(1, n + 1))


POINTERS = set("q k v q_out cache_layer positions page_table seq_lens node_counts freq status_dev out parents workspace tokens sampled pool path "
               "counts next_tokens new_lens uniforms temperature top_k top_p min_p".split())


def refused(lib, st, code, text=""):
    assert st == code, lib.dbt_last_error(None)
    assert text.encode() in lib.dbt_last_error(None)


def attn_args(**kw):
    a = dict(size=binding.ATTN_TREE_FORMAT.size, dtype=1, B=2, N=4, nq=8, nkv=4, D=128, pages=8, pps=4, scale=0.0, q=PTR, cache=PTR, s0=1, s1=1,
             s2=1, out=2 * PTR, table=PTR, lens=PTR, counts=0, parents=PTR, ws=PTR, ws_bytes=1 << 40, status=PTR)
    assert set(kw) <= set(a)
    a.update(kw)
    return binding.ATTN_TREE_FORMAT.pack(*a.values())


@pytest.mark.parametrize("change,code,text", [
    (dict(size=8), 1, "struct_size"), (dict(dtype=2), 2, "dtype"), (dict(B=0), 2, "B"), (dict(B=65536), 2, "B"), (dict(N=0), 2, "max_nodes"),
    (dict(N=65), 2, "max_nodes"), (dict(nq=6), 2, "multiple"), (dict(nq=0), 2, "multiple"), (dict(nq=68), 2, "16 query heads"), (dict(nkv=0), 2, "n_kv_heads"),
    (dict(D=96), 2, "head_dim"), (dict(pages=0), 1, "num_pages"), (dict(pages=1 << 26), 2, "2^26"), (dict(pps=0), 1, "pages_per_seq"),
    (dict(cache=0), 1, "NULL"), (dict(cache=PTR + 8), 1, "16-byte"), (dict(q=0), 1, "NULL"), (dict(out=0), 1, "NULL"), (dict(out=PTR), 1, "out must not be q"),
    (dict(out=PTR + 8), 1, "aligned"), (dict(q=PTR + 1), 1, "aligned"), (dict(parents=0), 1, "NULL"), (dict(table=0), 1, "NULL"), (dict(lens=0), 1, "NULL"),
    (dict(status=0), 1, "NULL"), (dict(ws=0), 1, "NULL"), (dict(ws=PTR + 16), 1, "256-byte"), (dict(ws_bytes=16), 3, "needed"),
    (dict(scale=-1.0), 1, "softmax_scale"), (dict(scale=math.nan), 1, "softmax_scale"), (dict(scale=math.inf), 1, "softmax_scale"),
])
def test_attn_tree_refusals(lib, change, code, text):
    refused(lib, lib.dbt_op_attn_tree(attn_args(**change), None), code, text)


def test_attn_tree_workspace_query(lib):
    n = C.c_size_t(0)
    assert lib.dbt_op_attn_tree_workspace(attn_args(q=0, cache=0, out=0, ws=0), C.byref(n)) == 0 and n.value > 0 and n.value % 256 == 0
    refused(lib, lib.dbt_op_attn_tree_workspace(attn_args(N=65), C.byref(n)), 2, "max_nodes")
    refused(lib, lib.dbt_op_attn_tree_workspace(attn_args(), None), 1, "NULL")
    refused(lib, lib.dbt_op_attn_tree_workspace(None, C.byref(n)), 1, "NULL")
    refused(lib, lib.dbt_op_attn_tree(None, None), 1, "NULL")


def append_args(**kw):
    a = dict(size=binding.ROPE_APPEND_FORMAT.size, dtype=1, B=2, N=4, nq=8, nkv=4, D=128, rot=128, inter=0, pages=8, pps=4, scale=1.0, q=PTR, k=PTR,
             v=PTR, a0=8, a1=8, a2=8, b0=8, b1=8, b2=8, c0=8, c1=8, c2=8, out=2 * PTR, cache=PTR, pos=PTR, table=PTR, lens=PTR, counts=0, freq=PTR,
             status=PTR)
    assert set(kw) <= set(a)
    a.update(kw)
    return binding.ROPE_APPEND_FORMAT.pack(*a.values())


@pytest.mark.parametrize("change,code,text", [
    (dict(size=8), 1, "struct_size"), (dict(dtype=-1), 2, "dtype"), (dict(N=65), 2, "max_nodes"), (dict(D=32), 2, "head_dim"), (dict(rot=0), 1, "rot_dim"),
    (dict(rot=63), 1, "rot_dim"), (dict(rot=130), 1, "rot_dim"), (dict(nq=0), 2, "n_q_heads"), (dict(q=0), 1, "NULL"), (dict(k=0), 1, "NULL"), (dict(v=0), 1, "NULL"),
    (dict(out=0), 1, "NULL"), (dict(out=PTR), 1, "q_out must not be q"), (dict(pos=0), 1, "NULL"), (dict(freq=0), 1, "NULL"), (dict(status=0), 1, "NULL"),
    (dict(cache=0), 1, "NULL"), (dict(k=PTR + 1), 1, "aligned"),
])
def test_rope_append_refusals(lib, change, code, text):
    refused(lib, lib.dbt_op_rope_append(append_args(**change), None), code, text)


def accept_args(**kw):
    a = dict(size=binding.TREE_ACCEPT_FORMAT.size, dtype=1, B=2, N=4, layers=2, nkv=4, D=128, pages=8, pps=4, tokens=PTR, parents=PTR, sampled=PTR,
             table=PTR, lens=PTR, counts=0, pool=PTR, path=2 * PTR, n=3 * PTR, follows=4 * PTR, new=5 * PTR, status=PTR)
    assert set(kw) <= set(a)
    a.update(kw)
    return binding.TREE_ACCEPT_FORMAT.pack(*a.values())


@pytest.mark.parametrize("change,code,text", [
    (dict(size=8), 1, "struct_size"), (dict(dtype=2), 2, "dtype"), (dict(layers=0), 2, "n_layers"), (dict(N=65), 2, "max_nodes"), (dict(tokens=0), 1, "NULL"),
    (dict(parents=0), 1, "NULL"), (dict(sampled=0), 1, "NULL"), (dict(pool=0), 1, "NULL"), (dict(path=0), 1, "NULL"), (dict(n=0), 1, "NULL"),
    (dict(follows=0), 1, "NULL"), (dict(new=0), 1, "NULL"), (dict(new=PTR), 1, "also an input"), (dict(path=PTR), 1, "also an input"), (dict(status=0), 1, "NULL"),
])
def test_tree_accept_refusals(lib, change, code, text):
    refused(lib, lib.dbt_op_tree_accept(accept_args(**change), None), code, text)


@pytest.mark.parametrize("change,code,text", [
    (dict(dtype=3), 2, "dtype"), (dict(rows=-1), 2, "rows"), (dict(vocab=1), 2, "vocab"), (dict(vocab=262145, stride=262145), 2, "vocab"),
    (dict(stride=99), 1, "row_stride"), (dict(logits=0), 1, "NULL"), (dict(u=0), 1, "NULL"), (dict(tokens=0), 1, "NULL"), (dict(logits=PTR + 2), 1, "aligned"),
])
def test_sample_refusals(lib, change, code, text):
    a = dict(logits=PTR, dtype=0, rows=2, vocab=100, stride=100, u=PTR, t=0, k=0, p=0, m=0, tokens=PTR, logprobs=0)
    a.update(change)
    refused(lib, lib.dbt_op_sample(*a.values(), None), code, text)


def test_sample_last_needs_a_handle(lib):
    assert lib.dbt_sample_last(None, None, 1, None, None) == 1


def test_sample_of_no_rows_is_nothing(lib):
    assert lib.dbt_op_sample(None, 0, 0, 100, 100, None, None, None, None, None, None, None, None) == 0


@pytest.mark.parametrize("change,code,text", [
    (dict(dtype=7), 2, "dtype"), (dict(rows=-1), 2, "rows"), (dict(heads=0), 2, "heads"), (dict(dim=1), 2, "head_dim"), (dict(rot=3), 1, "rot_dim"),
    (dict(rot=66), 1, "rot_dim"), (dict(x=0), 1, "NULL"), (dict(y=0), 1, "NULL"), (dict(pos=0), 1, "NULL"), (dict(freq=0), 1, "NULL"),
    (dict(y=PTR, ys=128), 1, "strides"), (dict(x=PTR + 2), 1, "aligned"),
])
def test_rope_refusals(lib, change, code, text):
    a = dict(x=PTR, y=2 * PTR, pos=PTR, freq=PTR, rows=4, heads=2, dim=64, rot=64, xs=256, xh=64, ys=256, yh=64, scale=1.0, inter=0, inv=0, dtype=0)
    a.update(change)
    refused(lib, lib.dbt_op_rope(*a.values(), None), code, text)


def test_rope_of_no_rows_is_nothing(lib):
    assert lib.dbt_op_rope(None, None, None, None, 0, 2, 64, 64, 128, 64, 128, 64, 1.0, 0, 0, 0, None) == 0


# ---- the binding's own checks -------------------------------------------------------------------------------------


def test_binding_refuses_cpu_tensors_and_wrong_shapes(lib):
    z, u = torch.zeros(2, 10), torch.zeros(2)
    for call in (lambda: binding.op_sample(z, u), lambda: binding.op_sample(z, u.double()), lambda: binding.op_sample(z, torch.zeros(3)),
                 lambda: binding.op_sample(z.t(), u), lambda: binding.op_sample(z.half(), u),
                 lambda: binding.op_sample(z, u, top_k=torch.zeros(2, dtype=torch.int64)),
                 lambda: binding.op_rope(torch.zeros(2, 3, 8), torch.zeros(2, dtype=torch.int32), torch.zeros(4, dtype=torch.float64)),
                 lambda: binding.op_rope(torch.zeros(2, 3, 8), torch.zeros(2, dtype=torch.int64), torch.zeros(4, dtype=torch.float64)),
                 lambda: binding.op_rope(torch.zeros(2, 3, 8), torch.zeros(2, dtype=torch.int32), torch.zeros(4))):
        with pytest.raises(binding.DbtError) as e:
            call()
        assert e.value.status == 1


def test_binding_refuses_caches_of_another_shape_or_type(lib):
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    q = torch.zeros(1, 2, 4, 64)
    for cache in (torch.zeros(2, 3, 2, 16, 128), torch.zeros(2, 3, 2, 8, 64), torch.zeros(3, 2, 16, 64), torch.zeros(2, 3, 2, 16, 64, dtype=torch.bfloat16)):
        with pytest.raises(binding.DbtError):
            binding.op_attn_tree(q, cache, i32(1, 2), i32(1), i32(1, 2))
    cache = torch.zeros(2, 3, 2, 16, 64)
    for kw in (dict(page_table=i32(2, 2)), dict(seq_lens=i32(2)), dict(parents=i32(1, 3)), dict(counts=i32(2)), dict(status=i32(3)),
               dict(out=torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16))):
        a = dict(page_table=i32(1, 2), seq_lens=i32(1), parents=i32(1, 2))
        a.update(kw)
        with pytest.raises(binding.DbtError):
            binding.op_attn_tree(q, cache, **a)


# ---- frequencies --------------------------------------------------------------------------------------------------


def test_plain_frequencies(lib):
    f, scale = binding.rope_frequencies(128, 10000.0)
    assert scale == 1.0 and f.shape == (64,)
    for i in (0, 1, 31, 63):
        assert f[i].item() == pytest.approx(10000.0 ** (-2 * i / 128), rel=1e-15)


def test_linear_and_base_frequencies(lib):
    f, scale = binding.rope_frequencies(64, 10000.0, "linear", factor=4.0)
    p, _ = binding.rope_frequencies(64, 10000.0)
    assert scale == 1.0 and torch.allclose(f * 4, p, rtol=1e-15, atol=0)
    f, scale = binding.rope_frequencies(64, 10000.0, "base", factor=4.0)
    assert scale == 1.0 and f[0] == 1.0 and f[-1].item() == pytest.approx(p[-1].item() / 4, rel=1e-12)
    assert (f[1:-1] < p[1:-1]).all() and (f[1:-1] > p[1:-1] / 4).all()


def test_ramp_frequencies(lib):
    f, scale = binding.rope_frequencies(128, 10000.0, "ramp", factor=16.0, trained_len=8192, low=1, high=32)
    p, _ = binding.rope_frequencies(128, 10000.0)
    assert scale == pytest.approx(0.1 * math.log(16) + 1, rel=1e-7)
    lo = math.floor(128 * math.log(8192 / (32 * 2 * math.pi)) / (2 * math.log(10000)))
    hi = math.ceil(128 * math.log(8192 / (2 * math.pi)) / (2 * math.log(10000)))
    for i in range(64):
        slow = min(1.0, max(0.0, (i - lo) / (hi - lo)))
        assert f[i].item() == pytest.approx(p[i].item() * (slow / 16 + 1 - slow), rel=1e-14)
    assert 0 < lo < hi < 63


@pytest.mark.parametrize("rot,base,trained,low,high", [(128, 10000.0, 131072, 1, 32), (128, 10000.0, 65536, 1, 32), (8, 10000.0, 8192, 1, 32), (64, 10000.0, 1e9, 1, 32),
                                                       (64, 10000.0, 1e14, 1, 2), (128, 10000.0, 8192, 1, 32), (128, 500000.0, 8192, 1, 32),
                                                       (64, 10000.0, 128, 1, 32), (64, 10000.0, 128, 32, 64), (64, 10000.0, 6, 1, 2), (2, 10000.0, 8192, 1, 32)])
def test_ramp_slows_each_pair_by_its_own_turns(lib, rot, base, trained, low, high):
    """Pairs of at most `low` turns slow by the whole factor and no others do, those of at least `high` keep; between them the ramp of
    the published method (YaRN, Peng et al. 2023), whose upper end is at most rot - 1: beyond the last pair where that one still makes
    more than `low` turns, and not cut to it."""
    factor = 16.0
    f, _ = binding.rope_frequencies(rot, base, "ramp", factor=factor, trained_len=trained, low=low, high=high)
    pair_of = lambda turns: rot * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
    lo, hi = max(math.floor(pair_of(high)), 0), min(math.ceil(pair_of(low)), rot - 1)
    for i in range(rot // 2):
        plain = base ** (-2 * i / rot)
        turns = trained * plain / (2 * math.pi)
        slow = 1.0 if i >= hi else 0.0 if i <= lo else (i - lo) / (hi - lo)
        assert f[i].item() == pytest.approx(plain * (slow / factor + 1 - slow), rel=1e-12)
        if turns <= low * (1 - 1e-12):
            assert f[i].item() == pytest.approx(plain / factor, rel=1e-12)
        elif turns >= high * (1 + 1e-12):
            assert f[i].item() == pytest.approx(plain, rel=1e-12)
        elif hi <= rot // 2 - 1:
            continue  # (the ramp's ends are whole pairs: the one below `low` turns may be the last, the one above `high` the first)
        else:
            assert f[i].item() > plain / factor * (1 + 1e-9)  # more than `low` turns, and the end lies behind it


def test_band_frequencies(lib):
    f, scale = binding.rope_frequencies(128, 500000.0, "bands", factor=8.0, trained_len=8192, low=1, high=4)
    p, _ = binding.rope_frequencies(128, 500000.0)
    assert scale == 1.0
    for i in range(64):
        turns = 8192 * p[i].item() / (2 * math.pi)
        keep = min(1.0, max(0.0, (turns - 1) / 3))
        assert f[i].item() == pytest.approx(p[i].item() * ((1 - keep) / 8 + keep), rel=1e-12)


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=64, base=1.0), dict(rot_dim=64, kind="linear", factor=0.5),
                                dict(rot_dim=64, kind="ramp", factor=2.0), dict(rot_dim=64, kind="bands", factor=2.0, trained_len=100, low=4, high=4),
                                dict(rot_dim=64, kind="ramp", factor=math.nan, trained_len=100), dict(rot_dim=2, kind="base", factor=2.0),
                                dict(rot_dim=64, kind="other")])
def test_frequency_refusals(lib, kw):
    with pytest.raises(binding.DbtError):
        binding.rope_frequencies(**kw)
