"""What the paged cache's entry points refuse, on the CPU: every check comes before anything is enqueued."""

import os
import subprocess

import pytest

from paper_2606_22327_amd import kvcache as C
from paper_2606_22327_amd import svfsim as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20     # an aligned address that nothing reads


def cache(**kw):
    f = dict(k=A, v=A, weight=A, position=A, kp=4096, kh=2048, kr=128, vp=4096, vh=2048, vr=128, num_pages=8,
             page_size=16, kv_heads=2, head_dim=128, dtype=0)
    f.update(kw)
    return C._CACHE.pack(*f.values())


def batch(**kw):
    f = dict(q_offsets=A, kv_len=A, page_table=A, table_stride=4, num_seqs=2, num_tokens=2, table_width=4, max_q=1)
    f.update(kw)
    return C._BATCH.pack(*f.values())


def append(**kw):
    f = dict(q=A, k=A, v=A, q_out=A, positions=A, rope=A, qt=1024, qh=128, kt=256, kh=128, vt=256, vh=128, ot=1024,
             oh=128, heads=8, rot=128, layout=0, rope_rows=10)
    f.update(kw)
    return C._APPEND.pack(*f.values())


def attend(**kw):
    f = dict(q=A, out=A, lse=A, workspace=A, workspace_bytes=1 << 40, qt=1024, qh=128, ot=1024, oh=128, scale=0.1,
             heads=8, causal=1, window=0, add_weight=0)
    f.update(kw)
    return C._ATTEND.pack(*f.values())


def evict(**kw):
    f = dict(next=A, new_len=2 * A, workspace=A, workspace_bytes=1 << 40, budget=32, recent=8, first=4)
    f.update(kw)
    return C._EVICT.pack(*f.values())


CACHE_BAD = [(dict(page_size=24), "page_size"), (dict(page_size=0), "page_size"), (dict(page_size=1 << 17), "page_size"),
             (dict(num_pages=-1), "num_pages"), (dict(kv_heads=0), "kv_heads"), (dict(head_dim=96), "head_dim"),
             (dict(dtype=2), "dtype"), (dict(num_pages=1 << 27), "2^31"), (dict(k=A + 8), "aligned"),
             (dict(v=0), "NULL"), (dict(kr=129), "multiples of 8"), (dict(vp=-8), "multiples of 8")]
BATCH_BAD = [(dict(num_seqs=-1), "num_seqs"), (dict(table_width=1 << 27, table_stride=1 << 27), "2^31"),
             (dict(table_stride=3), "table_stride"), (dict(kv_len=0), "NULL"), (dict(page_table=0), "NULL"),
             (dict(max_q=-1), "max_q")]


@pytest.mark.parametrize("fn,args", [("svf_kv_append", append), ("svf_kv_attend", attend), ("svf_kv_evict", evict)])
def test_cache_and_batch_are_checked_by_every_call(fn, args):
    call = getattr(S.load(), fn)
    for kw, text in CACHE_BAD:
        assert call(cache(**kw), batch(), args(), None) == -1, kw
        assert text in C.last_error(), (kw, C.last_error())
    for kw, text in BATCH_BAD:
        assert call(cache(), batch(**kw), args(), None) == -1, kw
        assert text in C.last_error(), (kw, C.last_error())
    for bad in ((None, batch(), args()), (cache(), None, args()), (cache(), batch(), None)):
        assert call(*bad, None) == -1
        assert "NULL" in C.last_error()


@pytest.mark.parametrize("kw,text", [
    (dict(heads=7), "multiple of kv_heads"), (dict(heads=0), "heads"), (dict(rot=7), "rot"), (dict(rot=130), "rot"),
    (dict(rot=-2), "rot"), (dict(layout=2), "layout"), (dict(rope=0), "table"), (dict(rope_rows=0), "table"),
    (dict(q=0), "NULL"), (dict(positions=0), "NULL"), (dict(qt=-1), "strides"), (dict(ot=2048), "in place"),
])
def test_append_refuses(kw, text):
    assert S.load().svf_kv_append(cache(), batch(), append(**kw), None) == -1
    assert text in C.last_error()


@pytest.mark.parametrize("kw,text", [
    (dict(heads=7), "multiple of kv_heads"), (dict(window=-1), "window"), (dict(scale=float("nan")), "scale"),
    (dict(out=A + 8), "aligned"), (dict(lse=0), "NULL"), (dict(oh=132), "multiples of 8"), (dict(qh=-1), "strides"),
])
def test_attend_refuses(kw, text):
    assert S.load().svf_kv_attend(cache(), batch(), attend(**kw), None) == -1
    assert text in C.last_error()


def test_attend_needs_weights_and_workspace():
    lib = S.load()
    assert lib.svf_kv_attend(cache(weight=0), batch(), attend(add_weight=1), None) == -1 and "weight" in C.last_error()
    need = lib.svf_kv_attend_workspace(cache(), batch(), attend(add_weight=1))
    assert need >= 0
    if need:
        assert lib.svf_kv_attend(cache(), batch(), attend(add_weight=1, workspace_bytes=need - 1), None) == -1
        assert "workspace" in C.last_error()
        assert lib.svf_kv_attend(cache(), batch(), attend(add_weight=1, workspace=A + 16), None) == -1
    assert lib.svf_kv_attend_workspace(cache(head_dim=3), batch(), attend()) == -1


@pytest.mark.parametrize("kw,text", [
    (dict(budget=0), "budget"), (dict(recent=-1), "budget"), (dict(first=25), "budget"), (dict(next=0), "NULL"),
    (dict(new_len=0), "NULL"), (dict(new_len=A), "must not be kv_len"), (dict(workspace=0), "workspace"), (dict(workspace_bytes=8), "workspace"),
])
def test_evict_refuses(kw, text):
    assert S.load().svf_kv_evict(cache(), batch(), evict(**kw), None) == -1
    assert text in C.last_error()


def test_evict_needs_weight_and_position():
    lib = S.load()
    assert lib.svf_kv_evict(cache(weight=0), batch(), evict(), None) == -1 and "weight" in C.last_error()
    assert lib.svf_kv_evict(cache(position=0), batch(), evict(), None) == -1 and "position" in C.last_error()
    # room for min(budget, slots over it) pairs of each key head
    assert lib.svf_kv_evict_workspace(cache(), batch(), evict()) == 256 + 4 * 32 * 8
    assert lib.svf_kv_evict_workspace(cache(), batch(), evict(budget=60)) == 256 + 4 * 4 * 8
    assert lib.svf_kv_evict_workspace(cache(), batch(), evict(budget=64)) == 256


def test_nothing_to_do_is_no_error():
    lib = S.load()
    assert lib.svf_kv_append(cache(), batch(num_tokens=0), append(), None) == 0
    assert lib.svf_kv_attend(cache(), batch(num_tokens=0), attend(), None) == 0
    assert lib.svf_kv_evict(cache(), batch(num_seqs=0), evict(), None) == 0


def test_structs_have_the_headers_layout(tmp_path):
    """The packed structs of the binding against the compiler's view of svfkv.h."""
    src = tmp_path / "layout.c"
    src.write_text("""#include <stdio.h>
#include <stddef.h>
#include "svfkv.h"
int main(void) {
    printf("%zu %zu %zu %zu %zu\\n", sizeof(svf_kv_cache), sizeof(svf_kv_batch), sizeof(svf_kv_append_args),
           sizeof(svf_kv_attend_args), sizeof(svf_kv_evict_args));
    printf("%zu %zu %zu %zu %zu\\n", offsetof(svf_kv_cache, dtype), offsetof(svf_kv_batch, max_q),
           offsetof(svf_kv_append_args, rope_rows), offsetof(svf_kv_attend_args, add_weight),
           offsetof(svf_kv_evict_args, first));
    return 0;
}
""")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    sizes, offs = (list(map(int, x.split())) for x in
                   subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    assert sizes == [x.size for x in (C._CACHE, C._BATCH, C._APPEND, C._ATTEND, C._EVICT)]
    assert offs == [100 - 4, 44, 124, 88, 40]


def test_binding_refuses_host_tensors_and_wrong_types():
    import torch
    k = torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16)
    b = C.Batch(torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32),
                torch.zeros((1, 4), dtype=torch.int32), 1)
    q = torch.zeros((1, 8, 128), dtype=torch.bfloat16)
    for cache_, text in ((C.Cache(k, k), "GPU"), (C.Cache(k.float(), k.float()), "bfloat16"),
                         (C.Cache(k, k[:2]), "shape"), (C.Cache(k.transpose(2, 3), k.transpose(2, 3)), "q")):
        with pytest.raises(S.SvfError) as e:
            C.attend(q.to(cache_.k.dtype), b, cache_)
        assert e.value.name == "SVF_EINVAL" and text in str(e.value)
    with pytest.raises(S.SvfError):
        C.rope_table(10, 7)
    with pytest.raises(S.SvfError):
        C.rope_table(10, 8, scaling="by-parts")
