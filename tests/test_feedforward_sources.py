"""Rules of the feed-forward kernels that no result shows, checked on their sources."""
import os
import re

from test_kernel_sources import CSRC, _code, _headers

FILES = ("rms_norm.cu", "gated_ffn.cu", "lora.cu", "tile_gemm.cuh", "skinny_gemm.cuh")


def test_no_read_only_loads_in_chained_kernels():
    """A chained kernel runs while the launch before it writes what it will read: a load through the read-only path may be moved above
    the wait, and asks for memory that nobody writes while the kernel runs."""
    for name in FILES:
        code = _code(name)
        assert "__ldg" not in code and "ld.global.nc" not in code and "__restrict__" not in code, name


# What a wait for earlier launches stands under, with the reason why nothing of theirs is touched without it.  `late`: a projection right behind
# the kernel that makes t, which lets it start only after its own wait has returned -- so x, W, bias, adapters and the requests' indices are there, and only
# t and the memory of the results have to be waited for.
WAITS = {
    "tile_gemm.cuh": {
        "if (!late)": 1,                                        # all threads, before anything is read
        "if (late && s0 + KSUB > p.k_main) ;": 1,               # producer: ahead of the first step that reads t
        "if (late)": 1,                                         # epilogue: ahead of the first store
    },
    "skinny_gemm.cuh": {
        "if constexpr (SHRINK)": 1,                             # t itself: all threads, before the adapter's index is read
        "if (!late)": 1,                                        # the others: all threads, before anything is read
        "if (late) ;": 1,                                       # producer: ahead of the first load of t
        "if (late)": 1,                                         # epilogue: ahead of t (single tokens) and of the closing barrier, behind which results are written
    },
}


def test_every_conditional_wait_of_the_product_headers_is_listed():
    for name in sorted(f for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))):
        if name == "sm100.cuh":
            continue                                            # (where it is defined)
        code, under = _code(name), {}
        for m in re.finditer(r"([^;{}]*)\bgrid_dep_wait\(\)", code):
            before = " ".join(m.group(1).split())
            head = before + " ;" if before else _headers(code, m.start(1))[0]
            under[head] = under.get(head, 0) + 1
        assert under == WAITS.get(name, {}), name


def test_the_next_launch_may_start_only_behind_a_wait_and_with_tensor_memory_in_hand():
    launches = 0
    for name in FILES:
        code = _code(name)
        for m in re.finditer(r"\bgrid_dep_launch\(\)", code):
            launches += 1
            statements = [" ".join(t.split()) for t in re.split(r"[;{}]", code[:m.start()])]
            assert statements[-1] in ("", "if (threadIdx.x == 0)", "if (et == 0)") and statements[-2] == "grid_dep_wait()", (name, statements[-2:])
            if name.endswith(".cuh"):
                body = code[code.rindex("extern __shared__", 0, m.start()):m.start()]
                assert "tmem_alloc(tmem_slot" in body and "__syncthreads()" in body[body.index("tmem_alloc(tmem_slot"):], name
    assert launches == 8


def test_what_waits_late_reads_nothing_of_t_before():
    tile, few = _code("tile_gemm.cuh"), _code("skinny_gemm.cuh")
    # tiles: t's map is read at one place, for steps behind K's own
    assert tile.count("maps.a2") == 1 and "if (s < p.k_main)" in tile[:tile.index("maps.a2")]
    # few tokens: t's map and pointer are read behind the producer's and the epilogue's waits
    load = few.index("&maps.t, &full")
    assert "if (late) grid_dep_wait();" in few[few.index("if (warp == 0) {"):load]
    use = few.index("p.t +")
    epilogue = few[few.index("const int quad = warp & 3"):]
    assert epilogue.index("grid_dep_wait()") < epilogue.index("p.t +") and few.count("p.t +") == 1 and use > load
    # nothing is stored before the epilogue has waited: stores stand behind a barrier of all threads
    assert few.index("store_bf16x8(p.") > few.rindex("__syncthreads()")
    assert tile.count("tma_store_3d(") == 1 and tile.index("if (late) {") < tile.index("tma_store_3d(")


def test_an_accumulator_is_released_only_where_a_later_tile_asks_for_it():
    """The odd CTA of a pair releases by an arrival on the even CTA's barrier: one that nobody waits for would be under way while the pair leaves."""
    tile = _code("tile_gemm.cuh")
    release = tile.index("mbar_arrive_cluster(mapa_shared(smem_u32(&tmem_empty[acc]), 0))")
    heads = _headers(tile, release)
    assert any(h.startswith("if (") and "tile + 2 * n_workers < total_tiles" in h for h in heads), heads
    # two accumulators in turn: the tile after the next is the one that asks
    assert "mbar_wait_cluster(&tmem_empty[acc], acc_phase ^ 1" in tile and tile.count("if (++acc == 2)") == 2


def _after(code, at):
    """The statement behind the one (or the block) that begins at `at`, which is an if."""
    depth, i = 0, code.index("(", at)
    while True:                                   # the condition
        depth += {"(": 1, ")": -1}.get(code[i], 0)
        i += 1
        if depth == 0:
            break
    while code[i].isspace():
        i += 1
    if code[i] == "{":
        depth = 0
        while True:
            depth += {"{": 1, "}": -1}.get(code[i], 0)
            i += 1
            if depth == 0:
                break
    else:
        i = code.index(";", i) + 1
    return " ".join(code[i:].split())


def test_whole_warps_meet_behind_what_one_lane_does():
    """tcgen05.ld, elect.sync, barrier.cluster and bar.red want all lanes of a warp at once: behind a branch that a single lane takes,
    __syncwarp() is the next thing that happens."""
    found = 0
    for name in ("tile_gemm.cuh", "skinny_gemm.cuh"):
        code = _code(name)
        code = code[:code.index("struct Shape {" if name == "tile_gemm.cuh" else "int launch_clusters(")]
        for m in re.finditer(r"\bif \((lane == 0|et == 0|threadIdx\.x == 0|(ok && )?elect_one\(\))\)", code):
            if "mbar_init" in code[m.end():m.end() + 120]:
                continue                          # the barriers' setup: __syncthreads() stands behind it, and warp 1's own work between
            found += 1
            rest = _after(code, m.start())
            assert re.match(r"(else mbar_arrive\(&tmem_empty\[acc\]\); |\+\+used; |\} )*__syncwarp\(\);", rest), (name, m.group(), rest[:80])
    assert found == 17
    # loops whose lanes leave at different rounds, ahead of a wait that a warp polls together
    few = _code("skinny_gemm.cuh")
    ahead = few[:few.index("const bool ok = aligned && mbar_wait_warp(done")]
    assert ahead.rstrip().endswith("__syncwarp();")


def test_a_wait_that_gives_up_is_reported_at_once():
    """... and not behind the closing barriers, which a CTA whose peer has stopped never passes: once in each role, ahead of anything that could wait."""
    for name, closing in (("tile_gemm.cuh", "// Neither CTA"), ("skinny_gemm.cuh", "// TMEM goes back")):
        raw = open(os.path.join(CSRC, name)).read()
        roles = raw[raw.index("TMA producer -"):raw.index(closing)]
        parts = re.split(r"// -+ (?:MMA issuer|epilogue)[^\n]*-", roles)
        assert len(parts) == 3
        for part in parts:
            code = re.sub(r"//[^\n]*", "", part)
            assert code.count("report_timeout(p.status)") == 1, name
            at = code.index("report_timeout(p.status)")
            assert "mbar_wait_slow" not in code[:at] and "bulk_wait<0>" not in code[:at], name
    helper = _code("sm100.cuh")
    assert "atomicExch(status, STATUS_TIMEOUT_MBARRIER)" in helper[helper.index("void report_timeout("):]
