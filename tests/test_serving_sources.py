"""Rules that the serving kernels' sources have to keep: dependent launch, tensor memory, registers that roles share out.
What breaks them is a wait that never ends or stale data, which no test provokes on a GPU."""
import os
import re

import pytest

from paper_2602_02071_b200 import build

SRC = {n: open(os.path.join(build.CSRC, n)).read() for n in sorted(os.listdir(build.CSRC)) if n.endswith((".cu", ".cuh"))}
CODE = {n: re.sub(r"//[^\n]*", "", s) for n, s in SRC.items()}
NEW = ["baps_attention_window.cuh", "baps_kv_append.cuh", "baps_kv_attention.cuh", "baps_kv_pages.cuh"]


def kernels():
    """(name, body) of every __global__ function of the serving files."""
    for n in NEW:
        for m in re.finditer(r"__global__\s+void\s+(?:__launch_bounds__\((?:[^()]|\([^()]*\))*\)\s*)?(\w+)\(", CODE[n]):
            yield m.group(1), CODE[n][m.start():CODE[n].index("\n}", m.start())]


KERNELS = dict(kernels())


def test_all_kernels_are_found():
    assert set(KERNELS) == {"window_attention_kernel", "kv_append_kernel", "kv_attention_kernel", "kv_join_kernel", "kv_fork_plan_kernel",
                            "kv_fork_rows_kernel", "kv_compact_count_kernel", "kv_compact_lists_kernel", "kv_compact_move_kernel"}
    assert sum(c.count("__global__") for n, c in CODE.items() if n in NEW) == len(KERNELS)


@pytest.mark.parametrize("name", sorted(KERNELS))
def test_every_kernel_waits_for_the_kernel_ahead_before_it_reads(name):
    body = KERNELS[name]
    assert body.count("await_previous_kernel(") == 1 and body.count("allow_next_kernel()") == 1
    wait = body.index("await_previous_kernel(")
    # no caller memory ahead of the wait: parameters are only read through pointers behind it
    assert not re.search(r"p\.\w+\s*\[|\*p\.|\*reinterpret_cast", body[body.index("{"):wait])


def test_tensor_memory_is_taken_between_the_kernel_ahead_and_the_next_one():
    body = KERNELS["window_attention_kernel"]
    assert body.index("await_previous_kernel()") < body.index("tmem_alloc(") < body.index("allow_next_kernel()") < body.index("tmem_dealloc(")
    # what three CTAs of an SM hold fits
    code = CODE["baps_attention_window.cuh"]
    assert re.search(r"kTmemCols = kKeys == 64 \? 128 : 256 \* kStreams", code) and re.search(r"kCtasPerSm = kKeys == 64 \? 3 : 1", code)


def test_the_cache_kernels_wait_for_nothing_but_their_own_copies():
    for name, body in KERNELS.items():
        if name != "window_attention_kernel":
            assert "mbar_" not in body and "while" not in body, name


def test_the_windowed_kernel_has_the_registers_that_its_roles_share_out():
    code = CODE["baps_attention_window.cuh"]
    assert re.findall(r'setmaxnreg\.\w+\.sync\.aligned\.u32 %0;" ::"n"\(kTcSplit\.(few|many)\)', code) == ["few", "many"]
    assert code.count("setmaxnreg.") == 2 and code.index("!has_registers_for<") < code.index("return launch_kernel(")
    build.build()
    log = open(os.path.join(os.path.dirname(build.LIB), "build.log")).read()
    used = re.findall(r"Compiling entry function '\w*window_attention_kernelI\w*Li128ELi2ELi128E\w*'.*?Used (\d+) registers", log, re.S)
    # 128 threads at 64 and 512 at 104 out of 640 at what the kernel was compiled to
    assert len(used) == 2 and all(128 * 64 + 512 * 104 <= 640 * int(r) for r in used)


def block_end(code, at):
    """Index behind the brace that closes the one at or behind ``at``."""
    depth, i = 0, code.index("{", at)
    while True:
        depth += {"{": 1, "}": -1}.get(code[i], 0)
        i += 1
        if depth == 0:
            return i


def test_all_ctas_of_a_cluster_reach_both_of_its_barriers():
    """The cluster form of kv_attention_kernel meets twice: when its parts are there, and when all have read them.  A CTA that left
    before would keep the others waiting, without a limit."""
    for name, body in KERNELS.items():
        assert body.count("cluster_sync()") == (2 if name == "kv_attention_kernel" else 0), name
    code = CODE["baps_kv_attention.cuh"]
    assert code.count("barrier.cluster.arrive") == code.count("barrier.cluster.wait") == 1          # both in cluster_sync itself
    assert sum(CODE[n].count("barrier.cluster") for n in NEW) == 2
    body = KERNELS["kv_attention_kernel"]
    # what the cluster form runs of it: without the other form's branch, and without the bodies of lambdas, whose returns are their own
    first = body.index("if constexpr (kClusters) {")
    other = block_end(body, first)
    assert body[other:].lstrip().startswith("else {")
    path = body[:other] + body[block_end(body, other):]
    while (at := re.search(r"= \[&?\]", path)) is not None:
        path = path[:at.start()] + path[block_end(path, at.start()):]
    ahead = path[:path.rindex("cluster_sync()")]
    assert "return" not in ahead and "break" not in ahead and "kClusters || w < w1;" in ahead
    # both barriers stand in the one block of the cluster form, at its top level, and the block ends with the kernel
    at = path.rindex("if constexpr (kClusters) {")
    block = path[at:block_end(path, at)]
    depth = 0
    depths = []
    for i, c in enumerate(block):
        depth += {"{": 1, "}": -1}.get(c, 0)
        if block.startswith("cluster_sync()", i):
            depths.append(depth)
    assert depths == [1, 1] and re.search(r"cluster_sync\(\);\s*return;\s*}$", block)
