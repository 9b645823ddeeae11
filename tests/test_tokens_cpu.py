"""Host side of the loss, embedding and dropout calls: argument structures, refusals that need no device, and the reference's
generator against the published known answers."""
import ctypes
import os
import re
import subprocess

import numpy as np

import paper_2512_14628_amd as pkg
from paper_2512_14628_amd import binding
from tests import ref_tokens as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_loss_arguments_have_the_layout_the_binding_fills(tmp_path):
    header = open(os.path.join(ROOT, "include", "hsadmm.h")).read()
    name, cls = "hsadmm_softmax_loss_args_t", binding._LossArgs
    fields = [f for f, _ in cls._fields_]
    src = ["#include <stdio.h>", "#include <stddef.h>", '#include "hsadmm.h"', "int main(void) {", '  printf("%%zu\\n", sizeof(%s));' % name]
    src += ['  printf("%%zu\\n", offsetof(%s, %s));' % (name, f) for f in fields]
    c, exe = tmp_path / "args.c", tmp_path / "args"
    c.write_text("\n".join(src + ["  return 0;", "}"]))
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(c), "-o", str(exe)])
    out = [int(x) for x in subprocess.check_output([str(exe)], text=True).split()]
    assert out == [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f in fields]
    body = header[:header.index("} %s;" % name)]
    body = re.sub(r"/\*.*?\*/", "", body[body.rindex("typedef struct {"):], flags=re.S)
    assert re.findall(r"([A-Za-z_0-9]+);", body) == fields
    # what the binding packs reads back field by field
    values = list(range(1, len(fields) + 1))
    values[fields.index("scale")] = 2.5
    a = cls.from_buffer_copy(binding._LOSS_PACK.pack(*values))
    assert [getattr(a, f) for f in fields] == values and binding._LOSS_PACK.size == ctypes.sizeof(cls)


def test_calls_without_a_plan_are_refused():
    lib = pkg.load_library()
    size = ctypes.c_size_t()
    assert lib.hsadmm_embedding(None, 0, None, 0, None, 32, 1, 1.0, None, 1, None) == -1
    assert lib.hsadmm_embedding_workspace(None, 0, 1, ctypes.byref(size)) == -1
    assert lib.hsadmm_embedding_gradient(None, 0, None, 32, 1, None, 1, 0, 1.0, 0, None, None, 0, None) == -1
    assert lib.hsadmm_dropout(None, None, 1, None, 1, None, 1, 1, 1, 0, 0.5, 1, 1, None, None) == -1
    assert lib.hsadmm_softmax_loss_workspace(None, 0, 1, 0, 1, ctypes.byref(size)) == -1
    args = binding._LossArgs()
    args.struct_bytes = ctypes.sizeof(binding._LossArgs)
    assert lib.hsadmm_softmax_loss(None, ctypes.byref(args)) == -1
    args.struct_bytes -= 8
    assert lib.hsadmm_softmax_loss(ctypes.c_void_p(1), ctypes.byref(args)) == -1      # another size: nothing is read from it
    assert lib.hsadmm_softmax_loss(ctypes.c_void_p(1), None) == -1


def test_generator_against_the_known_answers_of_its_publication():
    """Counter and key of zeros, and of ones in every bit (the known-answer file published with the method)."""
    assert [hex(int(x)) for x in ref.philox_words([0], 0, 0)[0]] == ["0x6627e8d5", "0xe169c58d", "0xbc57ac4c", "0x9b00dbd8"]
    ones = 2 ** 64 - 1
    assert [hex(int(x)) for x in ref.philox_words([ones], ones, ones)[0]] == ["0x408f276d", "0x41c83b0e", "0xa20bc7c6", "0x6d5451fd"]


def test_kept_elements_do_not_depend_on_where_the_count_starts():
    whole, factor = ref.dropout_kept(1000, 0.3, 11, 12)
    part, same = ref.dropout_kept(500, 0.3, 11, 12, first=123)
    assert np.array_equal(part, whole[123:623]) and factor == same
