"""What the scores of answers refuse, on the CPU: every check comes before anything is enqueued."""

import os
import subprocess

import pytest
import torch

from paper_2606_22327_amd import logprobs as L
from paper_2606_22327_amd import svfsim as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20     # an aligned address that nothing reads


def args(**kw):
    f = dict(logits=A, token=A, logprob=A, entropy=A, rank=A, top_logprob=A, top_index=A, workspace=A,
             workspace_bytes=1 << 40, row_stride=1000, scale=1.0, rows=4, vocab=1000, top=5, dtype=0, token_bytes=8)
    f.update(kw)
    return L._ARGS.pack(*f.values())


@pytest.mark.parametrize("kw,text", [
    (dict(rows=-1), "rows"), (dict(vocab=0), "vocab"), (dict(top=-1), "top"), (dict(top=65), "top"),
    (dict(vocab=4, top=5), "top"), (dict(dtype=3), "dtype"), (dict(token_bytes=2), "token_bytes"),
    (dict(row_stride=-1), "row_stride"), (dict(row_stride=1 << 41), "row_stride"), (dict(scale=0.0), "scale"),
    (dict(scale=-1.0), "scale"), (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"),
    (dict(scale=3e38), "scale"), (dict(scale=1e-45), "scale"),
    (dict(logits=0), "NULL"), (dict(token=0), "NULL"), (dict(rank=0), "NULL"), (dict(top_index=0), "NULL"),
    (dict(logits=A + 1), "aligned"), (dict(logits=A + 2, dtype=2), "aligned"), (dict(token=A + 4), "aligned"),
    (dict(vocab=(1 << 21) + 1), "vocab"), (dict(rows=1 << 26, top=32), "2^31"), (dict(rows=1 << 24, top=0), "rows"),
])
def test_score_refuses(kw, text):
    if kw.get("scale") == 1e-45:
        assert S.load().svf_logprob(args(rows=0, **kw), None) in (0, -1)    # the smallest there is: either
        return
    assert S.load().svf_logprob(args(**kw), None) == -1
    assert text in L.last_error()


def test_workspace_is_checked():
    lib = S.load()
    assert lib.svf_logprob(None, None) == -1 and "NULL" in L.last_error()
    assert lib.svf_logprob_workspace(args(top=99)) == -1
    need = lib.svf_logprob_workspace(args(rows=1, vocab=150000))
    assert need >= 0
    if need:
        for kw in (dict(workspace_bytes=need - 1), dict(workspace=A + 16), dict(workspace=0)):
            assert lib.svf_logprob(args(rows=1, vocab=150000, **kw), None) == -1 and "workspace" in L.last_error()


def test_nothing_to_do_is_no_error():
    assert S.load().svf_logprob(args(rows=0), None) == 0


def test_struct_has_the_headers_layout(tmp_path):
    src = tmp_path / "layout.c"
    src.write_text("""#include <stdio.h>
#include <stddef.h>
#include "svflogprob.h"
int main(void) {
    printf("%zu %zu %zu %zu %d\\n", sizeof(svf_logprob_args), offsetof(svf_logprob_args, row_stride),
           offsetof(svf_logprob_args, scale), offsetof(svf_logprob_args, token_bytes), SVF_LOGPROB_MOST_TOP);
    return 0;
}
""")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = list(map(int, subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()))
    assert got == [L._ARGS.size, 72, 80, 100, L.MOST_TOP]


def test_binding_refuses_host_tensors_and_wrong_types():
    x, t = torch.zeros((3, 10)), torch.zeros(3, dtype=torch.int64)
    for logits, token, text in ((x, t, "GPU"), (x.double(), t, "bfloat16"), (x[0], t, "rows, vocab")):
        with pytest.raises(S.SvfError, match=text) as e:
            L.score(logits, token)
        assert e.value.name == "SVF_EINVAL"
