"""The entry points of the paged cache reject bad arguments on the host, before anything is launched (no GPU needed)."""
import ctypes
import os

import pytest
import torch

import paper_2502_17599_amd as pkg
from paper_2502_17599_amd import _lib as L

INVALID, UNSUPPORTED, WORKSPACE = 1, 3, 4
FAKE = 0x100000   # never dereferenced: every case below fails validation


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pkg.library_path()):
        from paper_2502_17599_amd.build import build_library
        build_library()
    return pkg.load_library()


def test_struct_sizes_match_the_header(tmp_path):
    import shutil
    import subprocess
    cc = shutil.which("gcc")
    if cc is None:
        pytest.skip("no C compiler")
    names = {"meda_page_pool": L.MedaPagePool, "meda_page_params": L.MedaPageParams, "meda_rotary_params": L.MedaRotaryParams,
             "meda_append_params": L.MedaAppendParams, "meda_store_params": L.MedaStoreParams, "meda_paged_params": L.MedaPagedParams}
    src, exe = tmp_path / "sizes.c", tmp_path / "sizes"
    lines = ['#include <stdio.h>', '#include "meda.h"', "int main(void) {"]
    for n, s in names.items():
        lines.append(f'  printf("%zu\\n", sizeof({n}));')
        lines += [f'  printf("%zu\\n", offsetof({n}, {f[0]}));' for f in s._fields_]
    src.write_text("\n".join(lines + ["  return 0;", "}"]))
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run([cc, "-I", inc, str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    want = [x for s in names.values() for x in [ctypes.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]]
    assert got == want


def _pool(**kw):
    base = dict(n_pages=100, page_stride=0, n_kv_heads=2, head_dim=128, page_size=64, dtype=1, k_pages=FAKE, v_pages=FAKE,
                k_scales=None, v_scales=None)
    base.update(kw)
    return L.MedaPagePool(*[base[n] for n, _ in L.MedaPagePool._fields_])


def _params(cls, base, kw):
    base = dict(base, **kw)
    p = cls()
    for n, _ in cls._fields_:
        if n in base:
            if isinstance(base[n], tuple):
                getattr(p, n)[:] = base[n]
            else:
                setattr(p, n, base[n])
    return p


BAD_POOLS = [(dict(n_pages=0), INVALID), (dict(n_pages=1 << 31), UNSUPPORTED), (dict(n_kv_heads=0), INVALID),
             (dict(n_kv_heads=65536), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(page_size=24), UNSUPPORTED),
             (dict(page_size=8), UNSUPPORTED), (dict(page_size=512), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED),
             (dict(page_stride=100), INVALID), (dict(page_stride=2 * 64 * 128 + 4), INVALID), (dict(page_stride=-1), INVALID),
             (dict(k_pages=None), INVALID), (dict(v_pages=FAKE + 8), INVALID), (dict(dtype=2), INVALID),
             (dict(dtype=2, k_scales=FAKE, v_scales=FAKE + 2), INVALID)]


# ---- block tables
PAGES = dict(n_pages=100, n_rows=4, max_blocks=8, page_size=64, max_new=2)


def _update(lib, kw=None, ptrs=None, ws=None, ws_bytes=1 << 20):
    args = dict(lens=FAKE, n_new=FAKE + 4096, table=FAKE + 8192, ring=FAKE + 16384, state=FAKE + 32768, lens_out=FAKE,
                state_out=FAKE + 32768, slots=FAKE + 65536, granted=None)
    args.update(ptrs or {})
    p = _params(L.MedaPageParams, PAGES, kw or {})
    return lib.meda_page_update(ctypes.byref(p), *args.values(), FAKE if ws is None else ws, ws_bytes, None)


def test_page_update_refuses(lib):
    for kw, want in ((dict(n_pages=0), INVALID), (dict(n_rows=0), INVALID), (dict(max_blocks=0), INVALID), (dict(max_new=-1), INVALID),
                     (dict(rows_per_seq=-1), INVALID), (dict(rows_per_seq=3), INVALID), (dict(rows_per_seq=8), INVALID),
                     (dict(n_pages=1 << 31), UNSUPPORTED), (dict(page_size=20), UNSUPPORTED), (dict(n_rows=65537), UNSUPPORTED),
                     (dict(n_rows=65536, max_blocks=32768), UNSUPPORTED), (dict(max_blocks=1 << 25), UNSUPPORTED)):
        assert _update(lib, kw) == want, kw
    for name in ("lens", "n_new", "table", "ring", "state", "lens_out", "state_out", "slots"):
        assert _update(lib, ptrs={name: None}) == INVALID, name
        assert _update(lib, ptrs={name: FAKE + 2}) == INVALID, name
    assert _update(lib, ptrs=dict(lens_out=FAKE + 4)) == INVALID       # overlaps lens without being it
    assert _update(lib, ptrs=dict(state_out=FAKE + 32768 + 8)) == INVALID
    for name, at in (("lens_out", FAKE + 4096), ("granted", FAKE), ("granted", FAKE + 4096 + 8), ("slots", FAKE + 8192 + 64),
                     ("table", FAKE + 16384 + 256), ("state_out", FAKE + 65536)):
        assert _update(lib, ptrs={name: at}) == INVALID, (name, at)    # written arrays overlap nothing
    assert _update(lib, ws=FAKE + 16) == WORKSPACE and _update(lib, ws=0) == WORKSPACE
    assert _update(lib, ws_bytes=lib.meda_page_update_workspace_bytes(4) - 1) == WORKSPACE
    assert lib.meda_page_update_workspace_bytes(0) == 0 and lib.meda_page_update_workspace_bytes(-3) == 0
    assert lib.meda_page_update(None, *[FAKE] * 10, 1 << 20, None) == INVALID


# ---- rotary positions
ROT = dict(n_tokens=5, q_stride=(1024, 128), q_out_stride=(1024, 128), k_stride=(256, 128), k_out_stride=(256, 128), n_q_heads=8,
           n_k_heads=2, head_dim=128, rot_dim=128, n_axes=3, dtype=1)


def _rotary(lib, kw=None, ptrs=None):
    args = dict(q=FAKE, k=FAKE, positions=FAKE, inv_freq=FAKE, axis=FAKE, q_out=FAKE, k_out=FAKE)
    args.update(ptrs or {})
    p = _params(L.MedaRotaryParams, ROT, kw or {})
    return lib.meda_rotary(ctypes.byref(p), *args.values(), None)


def test_rotary_refuses(lib):
    for kw, want in ((dict(n_tokens=-1), INVALID), (dict(n_tokens=(1 << 26) + 1), UNSUPPORTED), (dict(n_q_heads=-1), INVALID),
                     (dict(n_q_heads=65535), UNSUPPORTED), (dict(head_dim=80), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),
                     (dict(rot_dim=0), INVALID), (dict(rot_dim=3), INVALID), (dict(rot_dim=130), INVALID), (dict(rot_dim=-2), INVALID),
                     (dict(n_axes=0), INVALID), (dict(n_axes=5), INVALID), (dict(flags=4), INVALID), (dict(pos_stride=-1), INVALID),
                     (dict(q_stride=(1028, 128)), INVALID), (dict(k_out_stride=(256, 129)), INVALID), (dict(k_stride=(-256, 128)), INVALID)):
        assert _rotary(lib, kw) == want, kw
    for name in ("q", "k", "positions", "inv_freq", "axis", "q_out", "k_out"):
        assert _rotary(lib, ptrs={name: None}) == INVALID, name
    for name, off in (("q", 8), ("k_out", 2), ("positions", 2), ("inv_freq", 4)):
        assert _rotary(lib, ptrs={name: FAKE + off}) == INVALID, name
    # rows that are written share no memory: a stride of zero, heads or tokens inside each other
    for out in ((0, 128), (1024, 0), (1024, 64), (512, 128), (128, 512), (640, 128), (128, 639 // 16 * 16)):
        assert _rotary(lib, dict(q_out_stride=out)) == INVALID, out
    assert lib.meda_rotary(None, *[FAKE] * 7, None) == INVALID
    assert _rotary(lib, dict(n_tokens=0)) == 0 and _rotary(lib, dict(n_q_heads=0, n_k_heads=0)) == 0   # nothing to do


# ---- appended tokens
APP = dict(n_tokens=5, q_stride=(1024, 128), q_out_stride=(1024, 128), k_stride=(256, 128), v_stride=(256, 128), n_q_heads=8,
           rot_dim=128, n_axes=3, dtype=1)


def _append(lib, kw=None, ptrs=None, pool=None):
    args = dict(q=FAKE, k=FAKE, v=FAKE, positions=FAKE, inv_freq=FAKE, axis=FAKE, slots=FAKE, q_out=FAKE)
    args.update(ptrs or {})
    p = _params(L.MedaAppendParams, APP, kw or {})
    return lib.meda_paged_append(ctypes.byref(_pool(**(pool or {}))), ctypes.byref(p), *args.values(), None)


def test_append_refuses(lib):
    for kw, want in BAD_POOLS:
        assert _append(lib, pool=kw) == want, kw
    for kw, want in ((dict(n_tokens=-1), INVALID), (dict(n_tokens=1 << 27), UNSUPPORTED), (dict(n_q_heads=-1), INVALID), (dict(dtype=0), UNSUPPORTED),
                     (dict(dtype=2), UNSUPPORTED), (dict(rot_dim=7), INVALID), (dict(rot_dim=256), INVALID), (dict(n_axes=0), INVALID),
                     (dict(flags=2), INVALID), (dict(slot_stride=-1), INVALID), (dict(v_stride=(256, 4)), INVALID)):
        assert _append(lib, kw) == want, kw
    assert _append(lib, pool=dict(dtype=0)) == UNSUPPORTED             # bf16 rows, fp32 pages
    for name in ("q", "k", "v", "positions", "inv_freq", "axis", "slots", "q_out"):
        assert _append(lib, ptrs={name: None}) == INVALID, name
    for name, off in (("q", 8), ("k", 4), ("v", 2), ("slots", 4), ("q_out", 8)):
        assert _append(lib, ptrs={name: FAKE + off}) == INVALID, name
    assert _append(lib, dict(n_tokens=0)) == 0


# ---- stored caches
STORE = dict(n_src_rows=1000, n_seqs=2, n_layers=3, max_blocks=8, dtype=1)


def _store(lib, kw=None, ptrs=None, pool=None):
    args = dict(k=FAKE, v=FAKE, layer_len=FAKE, layer_off=FAKE, lens=FAKE, table=FAKE)
    args.update(ptrs or {})
    p = _params(L.MedaStoreParams, STORE, kw or {})
    return lib.meda_paged_store(ctypes.byref(_pool(**(pool or {}))), ctypes.byref(p), *args.values(), None)


def test_store_refuses(lib):
    for kw, want in BAD_POOLS:
        assert _store(lib, pool=kw) == want, kw
    for kw, want in ((dict(n_src_rows=-1), INVALID), (dict(n_seqs=0), INVALID), (dict(n_layers=0), INVALID), (dict(max_blocks=0), INVALID),
                     (dict(n_seqs=70000), UNSUPPORTED), (dict(max_blocks=1 << 25), UNSUPPORTED), (dict(table_stride=7), INVALID),
                     (dict(table_stride=-8), INVALID), (dict(len_stride=-1), INVALID), (dict(dtype=0), UNSUPPORTED)):
        assert _store(lib, kw) == want, kw
    for name, off in (("k", 8), ("v", 8), ("layer_len", 2), ("layer_off", 4), ("lens", 2), ("table", 2)):
        assert _store(lib, ptrs={name: None}) == INVALID, name
        assert _store(lib, ptrs={name: FAKE + off}) == INVALID, name


# ---- attention
ATT = dict(n_rows=4, n_q_heads=8, max_blocks=8, dtype=1)


def _attend(lib, kw=None, ptrs=None, pool=None, ws=FAKE, short=0):
    args = dict(q=FAKE, table=FAKE, lens=FAKE, out=FAKE)
    args.update(ptrs or {})
    p, pl = _params(L.MedaPagedParams, ATT, kw or {}), _pool(**(pool or {}))
    need = lib.meda_paged_workspace_bytes(ctypes.byref(pl), ctypes.byref(p))
    return lib.meda_paged_attention(ctypes.byref(pl), ctypes.byref(p), *args.values(), ws, max(0, need - short) if need else 1 << 30, None)


def test_attention_refuses(lib):
    for kw, want in BAD_POOLS:
        assert _attend(lib, pool=kw) == want, kw
    for kw, want in ((dict(n_rows=0), INVALID), (dict(n_rows=65537), UNSUPPORTED), (dict(n_q_heads=0), INVALID), (dict(n_q_heads=7), INVALID),
                     (dict(n_q_heads=34), UNSUPPORTED), (dict(max_blocks=0), INVALID), (dict(max_blocks=1 << 25), UNSUPPORTED),
                     (dict(dtype=0), UNSUPPORTED), (dict(dtype=5), UNSUPPORTED), (dict(softmax_scale=-1.0), INVALID),
                     (dict(softmax_scale=float("nan")), INVALID), (dict(softmax_scale=float("inf")), INVALID),
                     (dict(q_stride=1000), INVALID), (dict(q_stride=1028), INVALID), (dict(out_stride=512), INVALID),
                     (dict(table_stride=7), INVALID), (dict(len_stride=-1), INVALID), (dict(q_stride=1 << 41), UNSUPPORTED)):
        assert _attend(lib, kw) == want, kw
        p, pl = _params(L.MedaPagedParams, ATT, kw), _pool()
        assert lib.meda_paged_workspace_bytes(ctypes.byref(pl), ctypes.byref(p)) == 0
    for name, off in (("q", 8), ("table", 2), ("lens", 1), ("out", 4)):
        assert _attend(lib, ptrs={name: None}) == INVALID, name
        assert _attend(lib, ptrs={name: FAKE + off}) == INVALID, name
    assert _attend(lib, ws=None) == WORKSPACE and _attend(lib, ws=FAKE + 64) == WORKSPACE and _attend(lib, short=1) == WORKSPACE


def test_workspace_is_bounded_and_a_multiple_of_256(lib):
    for rows, blocks, heads in ((1, 1, 2), (1, 100000, 32), (65536, 2000, 16)):
        p, pl = _params(L.MedaPagedParams, ATT, dict(n_rows=rows, max_blocks=blocks, n_q_heads=heads)), _pool()
        need = lib.meda_paged_workspace_bytes(ctypes.byref(pl), ctypes.byref(p))
        assert 0 < need < (32 << 20) and need % 256 == 0


def test_python_binding_refuses_on_the_host():
    """What the binding can see without a GPU."""
    cpu = torch.zeros(4, 2, 64, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="k_pages"):
        pkg.PagePool(cpu, cpu)
    with pytest.raises(ValueError, match="inv_freq"):
        pkg.RotaryPlan(torch.zeros(8, dtype=torch.float64))
    with pytest.raises(ValueError, match="q: expected"):
        pkg.meda_rotary(torch.zeros(3, 2, 64), None, None, None)
    with pytest.raises(ValueError, match="table"):
        pkg.meda_page_update(*[torch.zeros(4, dtype=torch.int32)] * 2, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32),
                             torch.zeros(2, dtype=torch.int64), 16)
