"""Paged cache and beam selection without a GPU: every refusal of the C entry
points, workspace sizes, and the page division."""
import ctypes

import pytest


def _pool(pb, **kw):
    p = pb.KvPool(0x1000, 2 * 4 * 16 * 64, 4 * 16 * 64, 16 * 64, 64, 10, 16, 4, 64)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


BAD_POOLS = [dict(base=0), dict(base=0x1008), dict(n_pages=0), dict(n_pages=(1 << 30) + 1), dict(page_size=0), dict(page_size=4097), dict(n_kv_heads=0),
             dict(head_dim=96), dict(page_stride=4), dict(page_stride=4100), dict(v_offset=-64), dict(head_stride=0),
             dict(token_stride=63), dict(token_stride=1 << 31), dict(token_stride=1 << 50),
             dict(head_stride=1 << 45)]
P = 0x10000  # a pointer that no refused call follows


def _append(pb, pool, dtype=1, k=P, ld_k=256, v=P, ld_v=256, n=8, tables=P, width=4, ld=4, start=P, lens=P, row0=P, S=2,
            rows=4):
    return pb.lib().pb_op_kv_append(dtype, k, ld_k, v, ld_v, n, ctypes.byref(pool) if pool else None, tables, width, ld,
                                    start, lens, row0, S, rows, None)


def _attend(pb, pool, dtype=0, q=P, ld_q=512, tables=P, width=4, ld=4, lens=P, S=2, H=8, scale=1.0, window=0, out=P,
            ld_out=512, ws=P, ws_bytes=64):
    return pb.lib().pb_op_paged_attention(dtype, q, ld_q, ctypes.byref(pool) if pool else None, tables, width, ld, lens, S,
                                          H, scale, window, 0, out, ld_out, ws, ws_bytes, None)


def _select(pb, logits=P, ld=100, scores=P, alive=P, B=2, W=3, V=100, eos=2, pad=1, o=(P, P, P, P), ws=P, ws_bytes=1 << 20):
    return pb.lib().pb_op_beam_select(logits, ld, scores, alive, B, W, V, eos, pad, *o, ws, ws_bytes, None)


def _fork(pb, pool, dtype=1, L=2, stride=1 << 20, parents=0x100000, R=4, tables=0x200000, width=8, lens=0x300000, S=4,
          refs=0x400000, grow=0x500000, ot=0x600000, os=0x700000, ol=0x800000, orf=0x900000, short=0xa00000, ws=0xb00000,
          ws_bytes=1 << 16):
    return pb.lib().pb_op_page_fork(dtype, ctypes.byref(pool) if pool else None, L, stride, parents, R, tables, width, lens,
                                    S, refs, grow, ot, os, ol, orf, short, ws, ws_bytes, None)


def _refused(pb, rc, what):
    assert rc == pb.PB_EINVAL, what
    assert pb.lib().pb_last_error().decode().startswith("pb_op_"), what


@pytest.mark.parametrize("bad", BAD_POOLS + [None], ids=str)
def test_pools_that_are_refused(bad):
    from paper_2503_17707_amd import binding as pb

    pool = None if bad is None else _pool(pb, **bad)
    _refused(pb, _append(pb, pool), bad)
    _refused(pb, _attend(pb, pool), bad)
    _refused(pb, _fork(pb, pool), bad)


def test_strides_of_single_places_do_not_matter():
    from paper_2503_17707_amd import binding as pb

    # refused for the missing operand, not for the pool
    for kw in (dict(n_pages=1, page_stride=-3), dict(page_size=1, token_stride=1), dict(n_kv_heads=1, head_stride=0)):
        assert _attend(pb, _pool(pb, **kw), lens=None) == pb.PB_EINVAL
        assert "lens" in pb.lib().pb_last_error().decode()


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(k=None), dict(v=P + 8), dict(ld_k=248), dict(ld_v=260), dict(n=-1),
                                 dict(tables=None), dict(width=0), dict(ld=3), dict(start=None), dict(lens=None),
                                 dict(S=-1), dict(S=65536), dict(rows=-1)], ids=str)
def test_append_refusals(bad):
    from paper_2503_17707_amd import binding as pb

    _refused(pb, _append(pb, _pool(pb), **bad), bad)


@pytest.mark.parametrize("bad", [dict(dtype=-1), dict(q=None), dict(q=P + 2), dict(ld_q=504), dict(ld_q=516), dict(out=None),
                                 dict(out=P + 8), dict(ld_out=256), dict(tables=None), dict(width=-1), dict(ld=2),
                                 dict(lens=None), dict(S=-2), dict(S=1 << 17), dict(H=0), dict(H=6), dict(H=1 << 17),
                                 dict(width=1 << 27, ld=1 << 27), dict(scale=float("nan")), dict(scale=float("inf")), dict(window=-1), dict(ws=P + 4)], ids=str)
def test_attention_refusals(bad):
    from paper_2503_17707_amd import binding as pb

    _refused(pb, _attend(pb, _pool(pb), **bad), bad)


def test_attention_of_more_blocks_than_a_launch_takes():
    from paper_2503_17707_amd import binding as pb

    far = dict(q=1 << 50, out=1 << 51, ld_q=1 << 16, ld_out=1 << 16, tables=1 << 44, lens=1 << 43, ws=None)
    for H, Hkv in ((256, 256), (257, 257), (4096, 256), (8192, 256), (8448, 256), (65520, 4), (1024, 128)):
        pool = _pool(pb, n_kv_heads=Hkv)
        fits = 65535 * Hkv * -(-(H // Hkv) // 32) < (1 << 24) - 8
        rc = _attend(pb, pool, S=65535, H=H, **dict(far, ld_q=H * 64, ld_out=H * 64, lens=None if fits else far["lens"]))
        _refused(pb, rc, (H, Hkv))
        assert ("lens" if fits else "blocks") in pb.lib().pb_last_error().decode(), (H, Hkv)


@pytest.mark.parametrize("bad", [dict(ws=P), dict(q=0x20000, ws=0x207f0), dict(out=0x20000, ws=0x1fff0),
                                 dict(out=0x20000, ld_out=1024, ws=0x20800), dict(lens=0x20004, ws=0x20000),
                                 dict(tables=0x20000, ld=400, ws=0x20640)], ids=str)
def test_attention_workspace_over_an_operand(bad):
    from paper_2503_17707_amd import binding as pb

    _refused(pb, _attend(pb, _pool(pb), **bad), bad)
    assert "overlap" in pb.lib().pb_last_error().decode()


@pytest.mark.parametrize("bad", [dict(logits=None), dict(logits=P + 2), dict(ld=99), dict(scores=None), dict(alive=None),
                                 dict(B=-1), dict(B=65536), dict(W=0), dict(W=33), dict(V=0), dict(V=(1 << 20) + 1, ld=1 << 21), dict(eos=-2),
                                 dict(eos=100), dict(pad=-1), dict(pad=100), dict(o=(None, P, P, P)), dict(o=(P, P, P, None)),
                                 dict(ws=None), dict(ws=P + 8), dict(ws_bytes=16)], ids=str)
def test_select_refusals(bad):
    from paper_2503_17707_amd import binding as pb

    _refused(pb, _select(pb, **bad), bad)


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(L=0), dict(stride=60), dict(stride=100), dict(parents=None), dict(R=-1),
                                 dict(R=65536), dict(tables=None), dict(width=0), dict(lens=None), dict(S=-1), dict(refs=None),
                                 dict(grow=None), dict(ot=None), dict(os=None), dict(ol=None), dict(orf=None),
                                 dict(short=None), dict(ws=None), dict(ws=0xb00004), dict(ws_bytes=8),
                                 dict(ot=0x200010), dict(ol=0x300000), dict(os=0x30000c), dict(orf=0x400000),
                                 dict(short=0x10000c), dict(ws=0x500000)], ids=str)
def test_fork_refusals(bad):
    from paper_2503_17707_amd import binding as pb

    _refused(pb, _fork(pb, _pool(pb), **bad), bad)


@pytest.mark.parametrize("bad", [dict(ol=0x700000), dict(os=0x60007c), dict(orf=0x600000), dict(short=0x80000c),
                                 dict(short=0x6ffffc), dict(ws=0x900020)], ids=str)
def test_fork_outputs_that_overlap(bad):
    from paper_2503_17707_amd import binding as pb

    _refused(pb, _fork(pb, _pool(pb), **bad), bad)
    assert "overlap" in pb.lib().pb_last_error().decode()


def test_fork_of_more_copies_than_a_launch_takes():
    from paper_2503_17707_amd import binding as pb

    # pages of 64 KB are two pieces; a page of a piece and a little, two
    far = dict(parents=0x10 << 32, tables=0x20 << 32, lens=0x30 << 32, grow=0x50 << 32, ot=0x60 << 32, os=0x70 << 32,
               ol=0x80 << 32, ws_bytes=1 << 22)
    _refused(pb, _fork(pb, _pool(pb, page_size=64), L=32768, R=32768, **far), "2^31")
    assert "2^31" in pb.lib().pb_last_error().decode()
    _refused(pb, _fork(pb, _pool(pb, page_size=33), L=32768, R=32768, **far), "2^31")
    assert "2^31" in pb.lib().pb_last_error().decode()


def test_nothing_to_do_is_no_error():
    from paper_2503_17707_amd import binding as pb

    pool = _pool(pb)
    assert _append(pb, pool, S=0) == 0 and _append(pb, pool, n=0) == 0 and _append(pb, pool, rows=0) == 0
    assert _attend(pb, pool, S=0) == 0
    assert _select(pb, B=0) == 0


def test_workspace_sizes():
    from paper_2503_17707_amd import binding as pb

    L = pb.lib()
    pool = _pool(pb)
    assert L.pb_op_beam_select_workspace(2, 4, 1000) > 0
    assert L.pb_op_beam_select_workspace(2, 0, 1000) == 0 and L.pb_op_beam_select_workspace(2, 4, 1 << 30) == 0
    assert L.pb_op_page_fork_workspace(4, 100) > 0 and L.pb_op_page_fork_workspace(-1, 100) == 0
    assert L.pb_op_paged_attention_workspace(2, 7, ctypes.byref(pool), 10) == 0
    assert L.pb_op_paged_attention_workspace(2, 8, None, 10) == 0


def test_page_division(tmp_path):
    """The quotients of page numbers against the machine's: divisors and numerators at
    the edges and between."""
    import os
    import shutil
    import subprocess

    if not shutil.which("g++"):
        pytest.skip("no C++ compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "div.cpp"
    src.write_text("""
#include <cstdio>
#include "fastdiv.h"
int main() {
    const uint32_t top = 0x7fffffffu;
    unsigned long long seed = 1;
    for (uint32_t k = 0; k < 20000; ++k) {
        seed = seed * 6364136223846793005ull + 1442695040888963407ull;
        const uint32_t d = k < 5000 ? k + 1 : k < 5031 ? 1u << (k - 5000) : k < 5062 ? (1u << (k - 5031)) + 1
                           : k < 5093 ? top >> (k - 5062) : (uint32_t)(seed >> 33) >> (k % 31);
        if (!d || d > top) continue;
        const pb::FastDiv f(d);
        for (int j = 0; j < 200; ++j) {
            seed = seed * 6364136223846793005ull + 1442695040888963407ull;
            const uint32_t q = (uint32_t)(seed >> 33) / d;
            const uint32_t ns[] = {(uint32_t)(seed >> 33), q * d, q * d + d - 1, q ? q * d - 1 : 0, top, (uint32_t)j};
            for (uint32_t n : ns)
                if (n <= top && f.quot(n) != n / d) return printf("%u / %u\\n", n, d), 1;
        }
    }
    return 0;
}
""")
    exe = str(tmp_path / "div")
    inc = os.path.join(root, "paper_2503_17707_amd", "paged")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I" + inc, str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_wrappers_refuse_what_the_library_cannot_see():
    import torch

    from paper_2503_17707_amd import binding as pb

    i32 = dict(dtype=torch.int32)
    pool = torch.zeros(6, 2, 4, 16, 64, dtype=torch.float16)
    k = torch.zeros(3, 4, 64, dtype=torch.float16)
    t, n = torch.zeros(3, 2, **i32), torch.zeros(3, **i32)
    q = torch.zeros(3, 8, 64, dtype=torch.float16)

    def refused(f, *a, **kw):
        with pytest.raises(pb.PbError) as e:
            f(*a, **kw)
        assert e.value.code == pb.PB_EINVAL

    # host tensors, wrong types, shapes and strides
    refused(pb.op_kv_append, 1, k, k, pool, t, n, n)
    refused(pb.op_kv_append, 0, k, k, pool, t, n, n)
    refused(pb.op_kv_append, 1, k, k[:, :2], pool, t, n, n)
    refused(pb.op_kv_append, 1, k, k, pool.transpose(3, 4), t, n, n)
    refused(pb.op_kv_append, 1, k, k, pool, t.long(), n, n)
    refused(pb.op_kv_append, 1, k, k, pool, t, n[:2], n)
    refused(pb.op_kv_append, 1, k, k, pool, t, n, n, row0=n.long())
    refused(pb.op_kv_append, 1, k.transpose(0, 1), k.transpose(0, 1), pool, t, n, n)
    refused(pb.op_paged_attention, 1, q, pool, t, n, q)
    refused(pb.op_paged_attention, 1, q[:2], pool, t, n, q[:2])
    refused(pb.op_paged_attention, 1, q, pool, t, n, q.float())
    refused(pb.op_paged_attention, 1, q, pool[:, :1], t, n, q)
    s, a = torch.zeros(2, 3), torch.zeros(2, 3, **i32)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    lg = torch.zeros(6, 50)
    refused(pb.op_beam_select, lg, s, a, s, a, a, a, eos=2, pad=1, workspace=ws)
    refused(pb.op_beam_select, lg.half(), s, a, s, a, a, a, eos=2, pad=1, workspace=ws)
    refused(pb.op_beam_select, lg[:5], s, a, s, a, a, a, eos=2, pad=1, workspace=ws)
    refused(pb.op_beam_select, lg, s, a.long(), s, a, a, a, eos=2, pad=1, workspace=ws)
    pools, r, sh = pool[None], torch.zeros(6, **i32), torch.zeros(2, **i32)
    refused(pb.op_page_fork, 1, pools, n, t, n, r, n, t, n, n, r, sh, ws)
    refused(pb.op_page_fork, 1, pool, n, t, n, r, n, t, n, n, r, sh, ws)
    refused(pb.op_page_fork, 1, pools, n, t, n, r[:5], n, t, n, n, r, sh, ws)
    refused(pb.op_page_fork, 1, pools, n, t, n, r, n, t[:2], n, n, r, sh, ws)
