"""CPU-side checks of the norms, the embeddings and the distillation loss: the layouts that the binding packs are the
header's, and null contexts and arguments are refused."""
import subprocess
from pathlib import Path

import pytest

import paper_2305_19982_b200 as adama
from paper_2305_19982_b200 import binding
from paper_2305_19982_b200 import build as adama_build

ROOT = Path(__file__).resolve().parent.parent
# struct, packing, fields in the header's order: p pointer, e enum or int, q 64-bit integer, d double
STRUCTS = [
    ("adama_distill_args", "_DISTILL_ARGS", "p:logits p:dlogits e:logits_dtype e:dlogits_dtype e:teacher_dtype e:top q:rows q:vocab"
     " q:ld_logits q:ld_dlogits q:ld_teacher q:ld_ids p:teacher_logits p:ids p:teacher_lse p:weights d:logit_scale p:loss p:stats"
     " p:workspace p:scratch"),
    ("adama_layer_norm_args", "_LAYER_NORM_ARGS", "p:x p:y e:x_dtype e:y_dtype q:rows q:dim q:ld_x q:ld_y p:weight p:bias d:eps p:mean p:rstd"),
    ("adama_layer_norm_backward_args", "_LAYER_NORM_BACKWARD_ARGS", "p:dy p:x p:dx e:dy_dtype e:x_dtype q:rows q:dim q:ld_dy q:ld_x"
     " q:ld_dx p:weight p:mean p:rstd p:dweight p:dbias p:m_weight p:v_weight p:m_bias p:v_bias p:workspace"),
    ("adama_embedding_args", "_EMBEDDING_ARGS", "p:ids p:table p:out e:table_dtype e:out_dtype q:tokens q:vocab q:dim q:ld_table q:ld_out d:scale"),
    ("adama_embedding_grad_args", "_EMBEDDING_GRAD_ARGS", "p:ids p:dy e:dy_dtype e:grad_dtype q:tokens q:vocab q:dim q:ld_dy q:ld_grad d:scale"
     " p:grad p:m p:v q:accumulate p:workspace"),
]


@pytest.fixture(scope="module")
def lib():
    adama_build.build()
    return adama.load_library()


@pytest.mark.parametrize("struct,packing,fields", STRUCTS, ids=[s[0] for s in STRUCTS])
def test_layouts_are_those_of_the_header(tmp_path, struct, packing, fields):
    fields = [f.split(":") for f in fields.split()]
    # 0 and 1 for the enums (their only values), other values all different
    values = [i + 0.25 if kind == "d" else (i % 2 if kind == "e" else i + 2) for i, (kind, _) in enumerate(fields)]
    show = {"p": "(double)(size_t)a.%s", "e": "(double)a.%s", "q": "(double)a.%s", "d": "a.%s"}
    lines = "\n".join('    printf("%%g\\n", %s);' % (show[kind] % name) for kind, name in fields)
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "adama.h"\nint main(void) {\n    %s a;\n'
                   "    if (fread(&a, 1, sizeof(a) + 1, stdin) != sizeof(a)) return 1;\n%s\n    return 0;\n}\n" % (struct, lines))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", str(ROOT / "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], input=getattr(binding, packing).pack(*values), capture_output=True, check=True).stdout.split()
    assert [float(x) for x in out] == [float(v) for v in values]


def test_null_contexts_are_refused(lib):
    bad = adama.Status.ERR_INVALID_ARG
    for name in ("distill_loss", "layer_norm", "layer_norm_backward", "embedding", "embedding_grad"):
        assert getattr(lib, "adama_" + name)(None, None, None) == bad
    for name in ("distill_scratch", "layer_norm_workspace", "embedding_workspace"):
        assert getattr(lib, "adama_" + name)(None, 16, 16) == 0
