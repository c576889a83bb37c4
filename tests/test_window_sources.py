"""What the tensor-core window kernels do around a bounded wait that gave up and around their status word, read from the source (no GPU: no
test makes a real kernel lose a signal)."""
import re

from test_giveup_sources import source

NAME = "psk_window_tc.cu"


def kernels():
    """{name: text} of the three kernels."""
    text = source(NAME)
    starts = [(m.start(), m.group(1)) for m in re.finditer(r"\n(tc_win_\w+_kernel)\(", text)]
    ends = [text.index("\n}\n", at) for at, _ in starts]
    found = {name: text[at:end] for (at, name), end in zip(starts, ends)}
    assert len(found) == 3
    return found


def test_the_status_word_is_cleared_where_no_cta_may_be_taken_over():
    """Any CTA that has not started may be taken over, the first one too: a kernel whose CTAs take items over leaves the clearing to one in front of it."""
    text = source(NAME)
    for name, body in kernels().items():
        clears = re.findall(r"[^\n]*\*status = 0;", body)
        assert all("!TAKES" in c for c in clears), name
        assert bool(clears) == (name != "tc_win_dkv_kernel"), name                 # (the key side follows the query side)
    for kernel, short in (("tc_win_fwd_kernel", "fwd"), ("tc_win_dq_kernel", "dq")):
        launch = text.index("launch_pdl(%s," % short)
        assert "takes ? %s<true> : %s<false>;" % (kernel, kernel) in text[launch - 400:launch] and "if (takes) clear_status(status, s);" in text[launch - 400:launch], kernel
    # and without items to take over nobody asks
    assert re.search(r"void sched_ask\([^)]*bool takes\) \{\s*if \(!takes\) return;", text)
    assert re.search(r"int sched_next\([^)]*bool takes[^)]*\) \{\s*if \(!takes \|\| ", text)


def test_a_later_wait_does_not_hide_one_that_gave_up():
    """`ok` is and-ed, or the next thing that happens is that the loop is left: at once, or after the warp's lanes agreed on it."""
    for name, body in kernels().items():
        waits = list(re.finditer(r"\bok = (?:ok && )?(?:__all_sync\(0xffffffff(?:u)?, )?(?:mbar_wait|sched_free)\([^;]*;", body))
        assert len(waits) >= 6, name
        for m in waits:
            stmt, after = m.group(0), body[m.end():].lstrip()
            anded = stmt.startswith("ok = ok && ") or stmt.endswith("&& ok;")
            agreed = re.match(r"ok = __all_sync\(0xffffffffu, ok\);\s*(?:if \(!ok\) (?:break|return);)", after)
            left = re.match(r"(?:\}\s*)?if \(!ok\) (?:break|return);", after)
            # the issuing lane: loops and statements that follow run only while `ok` holds
            guarded = re.match(r"\+\+items;\s*for \([^)]*&& ok;", after) or re.match(r"if \(t > 0\) ok = ok && ", after) or re.match(r"\+\+w\.done|owed = false", after)
            assert anded or agreed or left or guarded, (name, stmt, after[:120])


def test_no_copy_is_asked_for_after_a_wait_gave_up():
    """Between a wait of the loading warp and the loads behind it stands the way out."""
    for name, body in kernels().items():
        load = body[body.index("::kLoad) {"):body.index("::kMma) {", body.index("::kLoad) {"))]
        for m in re.finditer(r"mbar_wait\(", load):
            nxt = re.search(r"mbar_expect_tx\(|tma_load_4d\(|sched_ask\(|warp_load_tile<", load[m.end():])
            if nxt:
                assert re.search(r"if \(!ok\) (?:break|return);", load[m.end():m.end() + nxt.start()]), (name, load[m.start():m.start() + 80])


def test_finished_tiles_leave_only_without_a_wait_that_gave_up():
    for name, body in kernels().items():
        for m in re.finditer(r"tma_store_4d\(", body):
            assert "!cta_gave_up()" in body[body.rindex("if (", 0, m.start()):m.start()], name
        # rows formed again: behind the last barrier, where nobody waits any more
        last = body.rindex("__syncthreads();")
        assert body.index("redo_noted(") > last and "!cta_gave_up()" in body[last:body.index("redo_noted(")], name
        assert not re.search(r"redo_\w+_row|row_tainted|key_tainted", body[:last]), name


def test_tensor_memory_is_read_by_whole_warps():
    for name, body in kernels().items():
        for m in re.finditer(r"\bif \((?:[^{};]*\W)?ok\b[^{};]*\) \{", body):
            depth, i = 1, m.end()
            while depth:
                depth += {"{": 1, "}": -1}.get(body[i], 0)
                i += 1
            assert not re.search(r"\btmem_(?:ld|st)|stage_(?:row|half)\(|store_partial\(", body[m.end():i]), (name, m.group(0))


def roles(body):
    """(the loading warp's part, the issuing lane's)"""
    load = body.index("::kLoad) {")
    mma = body.index("::kMma) {", load)
    return body[load:mma], body[mma:body.index("} else {\n        const int ", mma)]


def test_the_feeding_warps_leave_their_loops():
    """A next answer or item would be met with `ok` formed anew."""
    for name, body in kernels().items():
        load, mma = roles(body)
        for part in (load, mma):
            assert all("&& ok" in h for h in re.findall(r"for \(int it = 0[^{}]*\) \{", part)), name
        assert re.search(r"if \(!ok\) break;\s*index = sched_next\(", mma), name
        if name == "tc_win_dq_kernel":                    # (asks for the next item's rows while it loads this one's keys)
            assert re.search(r"look_ahead\(\);\s*if \(!ok\) break;", load)
        else:
            assert re.search(r"if \(!ok\) break;\s*\}\s*index = sched_next\(", load), name
        # every lane of the loading warp goes the same way
        for m in re.finditer(r"\bok = (?:mbar_wait|sched_free)\([^;]*;", load):
            assert load[m.end():].lstrip().startswith("ok = __all_sync(0xffffffffu, ok);"), (name, m.group(0))


def test_no_mma_is_issued_after_a_wait_gave_up():
    for name, body in kernels().items():
        mma = roles(body)[1]
        for m in re.finditer(r"mbar_wait\(", mma):
            nxt = re.search(r"\bumma_\w+\(", mma[m.end():])
            if nxt:
                way = mma[m.end():m.end() + nxt.start()]
                assert re.search(r"if \(!ok\) (?:break|return);", way), (name, way)
