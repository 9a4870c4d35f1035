"""The operators for heads on a host without a GPU: the C ABI refuses before any
HIP call (made-up addresses are never read), the binding refuses host tensors,
and the plans of the kernels hold over their ranges."""
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2404_03617_amd as cf

needs_library = pytest.mark.skipif(not os.path.exists(cf.library_path()), reason="libconvfirst.so not built")
CSRC = os.path.join(os.path.dirname(cf.__file__), "csrc")

A, B, C1, C2, C3, S, OUT, O2, O3, O4, WS, G1, G2 = (i << 43 for i in range(1, 14))  # apart by more than any tensor
OK, INVALID, UNSUPPORTED, WORKSPACE = cf.CF_OK, cf.CF_ERR_INVALID, cf.CF_ERR_UNSUPPORTED, cf.CF_ERR_WORKSPACE
BIG = 1 << 40


def status_of(name, defaults, kw):
    v = dict(defaults)
    for k in kw:
        assert k in v, k
    v.update(kw)
    got = getattr(cf.lib(), name)(*v.values(), None)
    message = cf.lib().cf_last_error().decode()
    assert message.startswith(name + ": ") if got else message == "", message
    return got


NORM = dict(x=A, y=OUT, w=B, b=C1, stats=S, ws=WS, nbytes=BIG, N=3, P=50, C=64, G=8, ldx=64, ldy=64, eps=1e-6, dt=0,
            act=3)


@needs_library
@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(N=-1), INVALID), (dict(P=-1), INVALID),
    (dict(N=1 << 40, P=1 << 40), INVALID), (dict(C=0), INVALID), (dict(G=0), INVALID), (dict(G=7), INVALID),
    (dict(G=-8), INVALID), (dict(dt=2), INVALID), (dict(dt=-1), INVALID), (dict(act=4), INVALID),
    (dict(act=-1), INVALID), (dict(ldy=63), INVALID), (dict(ldx=-1), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(x=A + 1), INVALID),
    (dict(w=B + 2), INVALID), (dict(stats=S + 4), INVALID), (dict(y=A + 2), INVALID), (dict(y=A, ldy=65), INVALID),
    (dict(y=B), INVALID), (dict(stats=OUT), INVALID), (dict(C=8192, G=1, ldx=8192, ldy=8192), UNSUPPORTED),
    (dict(ldx=1 << 22), UNSUPPORTED), (dict(ldy=1 << 22), UNSUPPORTED),
    (dict(P=1 << 20, ws=None, nbytes=0), WORKSPACE), (dict(P=1 << 20, ws=WS + 8), INVALID),
    (dict(P=1 << 20, ws=A), INVALID), (dict(N=0, x=None, y=None), OK), (dict(P=0, x=None, y=None), OK),
])
def test_group_norm_forward_rejects(kw, status):
    assert status_of("cf_group_norm_forward", NORM, kw) == status


NORM_BACK = dict(dy=A, x=B, stats=S, w=C1, b=C2, dx=OUT, dw=O2, db=O3, ws=WS, nbytes=BIG, N=3, P=50, C=64, G=8,
                 lddy=64, ldx=64, lddx=64, dt=0, act=0)


@needs_library
@pytest.mark.parametrize("kw,status", [
    (dict(dy=None), INVALID), (dict(x=None), INVALID), (dict(stats=None), INVALID), (dict(dx=None), INVALID),
    (dict(dw=None), INVALID), (dict(db=None), INVALID), (dict(lddx=63), INVALID), (dict(lddy=-1), INVALID),
    (dict(dx=B), INVALID), (dict(dx=A, lddx=65), INVALID), (dict(db=O2), INVALID), (dict(dw=S), INVALID),
    (dict(stats=S + 4), INVALID), (dict(dw=O2 + 2), INVALID), (dict(act=9), INVALID), (dict(dt=2), INVALID),
    (dict(G=6), INVALID), (dict(C=8192, G=1, lddy=8192, ldx=8192, lddx=8192), UNSUPPORTED),
    (dict(lddy=1 << 22), UNSUPPORTED), (dict(ldx=1 << 22), UNSUPPORTED), (dict(lddx=1 << 22), UNSUPPORTED),
    (dict(ws=None, nbytes=0), WORKSPACE), (dict(nbytes=4), WORKSPACE), (dict(ws=WS + 4), INVALID),
    (dict(ws=O2), INVALID), (dict(N=0, dy=None, x=None, stats=None, dx=None, dw=None, db=None), OK),
])
def test_group_norm_backward_rejects(kw, status):
    assert status_of("cf_group_norm_backward", NORM_BACK, kw) == status


GATED = dict(x=A, wg=B, wu=C1, wd=C2, y=OUT, saved=S, ws=WS, nbytes=BIG, rows=50, C=64, H=96, ldx=64, ldg=64, ldu=64,
             ldd=96, ldy=64, dt=1, act=3)


@needs_library
@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INVALID), (dict(wg=None), INVALID), (dict(wu=None), INVALID), (dict(wd=None), INVALID),
    (dict(y=None), INVALID), (dict(rows=-1), INVALID), (dict(C=0), INVALID), (dict(H=0), INVALID), (dict(H=-4), INVALID),
    (dict(dt=2), INVALID), (dict(act=4), INVALID), (dict(ldx=-1), INVALID), (dict(ldg=-1), INVALID),
    (dict(ldu=-1), INVALID), (dict(ldd=-1), INVALID), (dict(ldy=63), INVALID), (dict(y=A), INVALID), (dict(y=C2), INVALID),
    (dict(saved=OUT), INVALID), (dict(saved=A), INVALID), (dict(saved=S + 2), INVALID), (dict(x=A + 1), INVALID),
    (dict(wd=C2 + 1), INVALID), (dict(ws=None, nbytes=0), WORKSPACE), (dict(nbytes=100), WORKSPACE),
    (dict(ws=WS + 8), INVALID), (dict(ws=OUT), INVALID), (dict(ws=C1), INVALID),
    (dict(rows=1 << 30), UNSUPPORTED), (dict(H=1 << 21, ldd=1 << 21), UNSUPPORTED),
    (dict(C=1 << 21, ldx=1 << 21, ldg=1 << 21, ldu=1 << 21, ldy=1 << 21), UNSUPPORTED),
    (dict(rows=0, x=None, y=None, wg=None, ws=None, nbytes=0), OK),
])
def test_gated_forward_rejects(kw, status):
    assert status_of("cf_gated_ffn_forward", GATED, kw) == status


GATED_BACK = dict(dy=A, x=B, saved=S, wg=C1, wu=C2, wd=C3, dx=OUT, dwg=O2, dwu=O3, dwd=O4, ws=WS, nbytes=BIG, rows=50,
                  C=64, H=96, lddy=64, ldx=64, ldg=64, ldu=64, ldd=96, lddx=64, dt=1, act=3)


@needs_library
@pytest.mark.parametrize("kw,status", [
    (dict(dy=None), INVALID), (dict(x=None), INVALID), (dict(saved=None), INVALID), (dict(wg=None), INVALID),
    (dict(wu=None), INVALID), (dict(wd=None), INVALID), (dict(dx=None), INVALID), (dict(dwg=None), INVALID),
    (dict(dwu=None), INVALID), (dict(dwd=None), INVALID), (dict(dx=A), INVALID), (dict(dwg=O3), INVALID),
    (dict(dwd=C3), INVALID), (dict(dwu=S), INVALID), (dict(lddx=63), INVALID), (dict(ldd=-1), INVALID),
    (dict(act=-1), INVALID), (dict(ws=None, nbytes=0), WORKSPACE), (dict(ws=WS + 8), INVALID), (dict(ws=O4), INVALID),
    (dict(rows=1 << 30), UNSUPPORTED), (dict(rows=0, dwg=None), INVALID),
])
def test_gated_backward_rejects(kw, status):
    assert status_of("cf_gated_ffn_backward", GATED_BACK, kw) == status


LINEAR = dict(x=A, w=B, tokens=C1, logp=OUT, lse=O2, ws=WS, nbytes=BIG, rows=50, C=64, V=1000, ldx=64, ldw=64, dt=0)


@needs_library
@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(lse=None), INVALID), (dict(tokens=None), INVALID),
    (dict(logp=None), INVALID), (dict(rows=-1), INVALID), (dict(C=0), INVALID), (dict(V=0), INVALID), (dict(dt=2), INVALID),
    (dict(ldx=-1), INVALID), (dict(ldw=-1), INVALID), (dict(tokens=C1 + 4), INVALID), (dict(x=A + 1), INVALID),
    (dict(lse=O2 + 2), INVALID), (dict(lse=OUT), INVALID), (dict(logp=C1), INVALID), (dict(lse=B), INVALID),
    (dict(ws=None, nbytes=0), WORKSPACE), (dict(ws=WS + 8), INVALID), (dict(ws=A), INVALID),
    (dict(rows=1 << 30), UNSUPPORTED), (dict(C=1 << 21, ldx=1 << 21, ldw=1 << 21), UNSUPPORTED),
    (dict(rows=0, x=None, w=None, lse=None, ws=None, nbytes=0), OK),
])
def test_linear_log_probs_forward_rejects(kw, status):
    assert status_of("cf_linear_log_probs_forward", LINEAR, kw) == status


LINEAR_BACK = dict(x=A, w=B, tokens=C1, logp=C2, lse=S, gl=G1, gs=G2, dx=OUT, dw=O2, ws=WS, nbytes=BIG, rows=50, C=64, V=1000,
                   ldx=64, ldw=64, lddx=64, dt=0)


@needs_library
@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(lse=None), INVALID), (dict(dx=None), INVALID),
    (dict(dw=None), INVALID), (dict(gl=None, gs=None), INVALID), (dict(tokens=None), INVALID), (dict(logp=None), INVALID), (dict(lddx=63), INVALID),
    (dict(logp=C2 + 2), INVALID), (dict(dx=C2), INVALID),
    (dict(dx=A), INVALID), (dict(dw=B), INVALID), (dict(dw=OUT), INVALID), (dict(dx=G1), INVALID),
    (dict(gs=G2 + 2), INVALID), (dict(ws=None, nbytes=0), WORKSPACE), (dict(ws=WS + 8), INVALID),
    (dict(ws=O2), INVALID), (dict(rows=1 << 30), UNSUPPORTED), (dict(rows=0, dw=None), INVALID),
])
def test_linear_log_probs_backward_rejects(kw, status):
    assert status_of("cf_linear_log_probs_backward", LINEAR_BACK, kw) == status


@needs_library
def test_launches_of_more_than_32_bits_are_refused():
    """Rows, classes and images whose launches would have 2^32 threads."""
    big = dict(C=8, ldx=8, ldw=8)
    assert status_of("cf_linear_log_probs_forward", LINEAR, dict(rows=1, V=1 << 28, **big)) == UNSUPPORTED
    assert status_of("cf_linear_log_probs_forward", LINEAR, dict(rows=1 << 28, V=10, **big)) == UNSUPPORTED
    big["lddx"] = 8
    assert status_of("cf_linear_log_probs_backward", LINEAR_BACK, dict(rows=1 << 28, V=10, **big)) == UNSUPPORTED
    assert status_of("cf_group_norm_forward", NORM, dict(N=1 << 25, P=1, G=64)) == UNSUPPORTED
    assert cf.lib().cf_linear_log_probs_workspace_bytes(1, 8, (1 << 28) - 1, 1) > 0


@needs_library
def test_silu_is_of_these_operators_alone():
    """The activations of training keep their list."""
    assert cf.lib().cf_act_forward(A, B, C1, C2, None, None, 4, 70, 70, 70, 0, 3, None) == INVALID


@needs_library
def test_workspace_queries():
    """0 for what has no kernel, room for what the formulas keep there (h, its
    gradients, a piece of dz), and without alignment for copies of the inputs too
    (which are there with it where rows are no multiple of 8 long; up to 16 rows of a
    forward call need none)."""
    L = cf.lib()
    assert L.cf_group_norm_workspace_bytes(2, 100, 64, 7) == 0
    assert L.cf_group_norm_workspace_bytes(2, 100, 8192, 1) == 0
    assert L.cf_group_norm_workspace_bytes(-1, 100, 64, 8) == 0
    assert L.cf_group_norm_backward_workspace_bytes(5, 100, 64, 8) >= 5 * 64 * 8
    for rows, C, H in ((1, 64, 96), (300, 100, 77), (5000, 512, 1365), (8192, 4096, 12288)):
        for f, least in ((L.cf_gated_ffn_workspace_bytes, 2), (L.cf_gated_ffn_backward_workspace_bytes, 6)):
            tight, loose = f(rows, C, H, 1), f(rows, C, H, 0)
            copied = C % 8 == 0 and H % 8 == 0 and (rows > 16 or least == 6)
            assert tight >= least * rows * H and loose >= tight + copied * 2 * (rows * C + 3 * C * H), (rows, C, H)
    for rows, C, V in ((1, 64, 1000), (300, 100, 77), (2047, 1000, 50021), (8192, 4096, 131072)):
        for f in (L.cf_linear_log_probs_workspace_bytes, L.cf_linear_log_probs_backward_workspace_bytes):
            tight, loose = f(rows, C, V, 1), f(rows, C, V, 0)
            copied = C % 8 == 0 and (rows > 16 or f == L.cf_linear_log_probs_backward_workspace_bytes)
            assert tight > 0 and loose >= tight + copied * 2 * (rows * C + V * C), (rows, C, V)
    dz = L.cf_linear_log_probs_backward_workspace_bytes(8192, 4096, 131072, 1)
    assert dz < 2 << 30  # the logits alone would be 2 GiB
    for f in (L.cf_gated_ffn_workspace_bytes, L.cf_linear_log_probs_workspace_bytes,
              L.cf_gated_ffn_backward_workspace_bytes, L.cf_linear_log_probs_backward_workspace_bytes):
        assert f(0, 64, 64, 1) == 0 and f(4, 0, 64, 1) == 0 and f(4, 64, -1, 1) == 0 and f(1 << 31, 64, 64, 1) == 0


@pytest.fixture
def no_library(monkeypatch):
    def fail():
        raise AssertionError("the library must not be reached")

    monkeypatch.setattr(cf, "lib", fail)


def test_host_tensors_and_other_types_are_refused(no_library):
    x, w, d = torch.zeros(4, 64, dtype=torch.float16), torch.zeros(96, 64, dtype=torch.float16), None
    d = torch.zeros(64, 96, dtype=torch.float16)
    t, s = torch.zeros(4, dtype=torch.int64), torch.zeros(4, 192)
    lp = cf.LinearLogProbs(torch.zeros(4), torch.zeros(4))
    for call in (lambda: cf.group_norm_forward(x, 8), lambda: cf.group_norm_forward_save(x, 8),
                 lambda: cf.group_norm_backward(x, x, torch.zeros(4, 8, 2)), lambda: cf.gated_ffn_forward(x, w, w, d),
                 lambda: cf.gated_ffn_forward_save(x, w, w, d), lambda: cf.gated_ffn_backward(x, x, s, w, w, d),
                 lambda: cf.linear_log_probs_forward(x, w, t),
                 lambda: cf.linear_log_probs_backward(x, w, t, lp, torch.zeros(4))):
        with pytest.raises(ValueError, match="GPU"):
            call()
    for call in (lambda: cf.group_norm_forward([1.0], 1), lambda: cf.gated_ffn_forward(None, w, w, d),
                 lambda: cf.linear_log_probs_forward("features", w)):
        with pytest.raises(TypeError):
            call()


def test_the_copies_of_gelus_tail_agree():
    """act(u) and act'(u) of the heads (cf_act.h), GELU (cf_device.h) and its slope
    (cf_ckpt.hip) evaluate the same q(t)."""

    def coefficients(name):
        text = open(os.path.join(CSRC, name)).read()
        at = text.index("-0.129858347f")
        return re.findall(r"-?0\.\d+f", text[at:text.index("exp2f", at)])

    want = coefficients("cf_device.h")
    assert len(want) >= 6 and coefficients("cf_act.h") == want == coefficients("cf_ckpt.hip")


# ---------------------------------------------------------------------------
# Plans


def run_cpp(tmp_path, header, namespace, body):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ not found")
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text('#include "%s"\n#include <initializer_list>\n#include <stdio.h>\nusing namespace cf::%s;\nint main() {\n%s\nreturn 0;\n}\n'
                   % (header, namespace, body))
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout[-2000:]
    return r.stdout


@pytest.mark.parametrize("cus", [256, 80])
def test_splits_of_the_products_hold_all_steps_and_fit_the_room(tmp_path, cus):
    """No split is empty, together they are all steps, one alone is never split
    where it may not be, and the partial sums fit."""
    run_cpp(tmp_path, "cf_mm_plan.h", "mm", """
    const int64_t sizes[] = {0, 1, 7, 64, 129, 1000, 4096, 12288, 131072, 1 << 20};
    for (int64_t M : sizes)
        for (int64_t N : sizes)
            for (int64_t steps = 0; steps < 1 << 22; steps += steps / 2 + 1)
                for (int batch = 1; batch < 3; batch++)
                    for (int split = 0; split < 2; split++) {
                        const Plan p = plan_of(M, N, steps, batch, split, %d, M %% 3 == 0 ? STORE : M %% 3 == 1 ? MORE : GATE);
                        const bool ok = p.tile >= 0 && p.tile < TILE_COUNT && p.splits >= 1 && p.per >= 1 &&
                                        (int64_t)p.splits * p.per >= steps && (split || p.splits == 1) &&
                                        (p.splits == 1 || (int64_t)(p.splits - 1) * p.per < steps) &&
                                        (double)part_bytes(p, M, N, batch) <= PART_BYTES;
                        if (!ok) {
                            printf("%%lld x %%lld, %%lld steps: tile %%d, %%d splits of %%d\\n", (long long)M, (long long)N,
                                   (long long)steps, p.tile, p.splits, p.per);
                            return 1;
                        }
                    }
    """ % cus)


@pytest.mark.parametrize("cus", [256, 80])
def test_no_split_of_a_launched_product_is_empty(tmp_path, cus):
    """What the kernel of a gradient's product over the classes is given, for each
    piece of the vocabulary, the last and shortest among them, by the plan for whole
    ones: every split begins before the last step (its reads would be behind the
    weights), together they are all steps, and their sums have room."""
    run_cpp(tmp_path, "cf_mm_plan.h", "mm", """
    int shorter = 0;
    const int64_t rows_of[] = {1, 16, 17, 40, 922, 4096, 8192, 20000, 32768, 50000, 262144};
    const int columns[] = {8, 16, 24, 64, 256, 512, 1000, 1024, 4096};
    for (int64_t rows : rows_of)
        for (int C : columns)
            for (int64_t V = 1; V < (1 << 28); V += V / 37 + 1) {
                const Pieces cut = pieces_of(rows, (int)V);
                const bool lo = in_parts(rows);
                const int64_t M = lo ? 2 * rows : rows;
                const Plan p = plan_of(M, C, steps_of(cut.columns), 1, true, %d);
                const int last = (int)(V - (int64_t)(cut.count - 1) * cut.columns);
                if (last < 1 || last > cut.columns) {
                    printf("%%lld rows, %%lld classes: the last piece has %%d\\n", (long long)rows, (long long)V, last);
                    return 1;
                }
                for (int n : {cut.columns, last}) {
                    const Args a = args_of(p, (int)M, C, n, Matrix{}, 0, Matrix{}, 0);
                    shorter += a.splits < p.splits;
                    if (a.splits < 1 || (int64_t)(a.splits - 1) * a.per >= a.steps || (int64_t)a.splits * a.per < a.steps ||
                        a.splits > p.splits || a.items != (unsigned)(a.tiles_m * a.tiles_n * a.splits)) {
                        printf("%%lld rows of %%d, a piece of %%d of %%lld: %%d splits of %%d, %%d steps\\n", (long long)rows, C, n,
                               (long long)V, a.splits, a.per, a.steps);
                        return 1;
                    }
                }
            }
    if (!shorter)
        return 1;
    // and for one plan, products of any length up to its own
    const Plan p = {1, 7, 13};
    for (int K = 0; K <= 7 * 12 * STEP; K += 5)
        for (int two = 0; two < 2; two++) {
            const Args a = args_of(p, 100, 100, two ? K / 2 : K, Matrix{}, 0, Matrix{}, 0, two);
            if (a.splits < 1 || (a.steps > 0 && (a.splits - 1) * a.per >= a.steps) || a.splits * a.per < a.steps)
                return 1;
        }
    """ % cus)


def test_both_tiles_and_splits_are_chosen(tmp_path):
    """Few tiles over a long axis are split, a chip full of large ones is not."""
    out = run_cpp(tmp_path, "cf_mm_plan.h", "mm", "".join(
        'p = plan_of(%d, %d, %d, 1, true, 256); printf("%%d %%d\\n", p.tile, p.splits);\n' % s
        for s in ((8192, 8192, 64), (512, 512, 400), (130, 200, 1), (8192, 4096, 192)))
        .replace("p = plan_of(8192, 8192", "Plan p = plan_of(8192, 8192", 1))
    rows = [tuple(int(v) for v in line.split()) for line in out.split("\n") if line]
    assert rows[0] == (0, 1) and rows[1][1] > 1 and rows[2] == (1, 1) and rows[3] == (0, 1)


@pytest.mark.parametrize("cus", [256, 80])
def test_parts_of_a_group_norm_hold_all_pixels_and_groups(tmp_path, cus):
    """Where there is a kernel, a workgroup's threads hold its channels, its parts
    are all of the pixels, none is empty, and a thread's vectors fit its registers;
    its groups are all groups."""
    run_cpp(tmp_path, "cf_gnorm_plan.h", "gnorm", """
    const int channels[] = {1, 2, 3, 8, 24, 64, 96, 100, 363, 512, 1000, 4096, 65536};
    for (int C : channels)
        for (int G = 1; G <= C; G++) {
            if (C %% G || C / G > 4096)
                continue;
            for (int64_t P = 1; P < 1 << 24; P += P / 2 + 1)
                for (int64_t N = 1; N < 3000; N *= 7)
                    for (int most : {FORWARD_NV, BACKWARD_NV}) {
                        const Plan p = plan_of(N, P, C, G, most, %d);
                        if (p.rows < 1)
                            continue;
                        const bool ok = p.per_block * p.blocks >= G && p.per_block * (p.blocks - 1) < G &&
                                        p.V * 8 >= p.per_block * (C / G) && p.rows * p.V <= p.threads && p.chunks >= 1 &&
                                        p.chunks * p.px >= P && (p.chunks - 1) * p.px < P && p.nv >= 1 && p.nv <= most &&
                                        (int64_t)p.nv * p.rows >= p.px;
                        if (!ok) {
                            printf("N %%lld P %%lld C %%d G %%d: %%d blocks, %%d chunks, nv %%d\\n", (long long)N, (long long)P, C, G,
                                   p.blocks, p.chunks, p.nv);
                            return 1;
                        }
                    }
        }
    """ % cus)


@pytest.mark.parametrize("cus", [256, 80])
def test_the_kernel_of_a_group_norm_holds_every_pixel(tmp_path, cus):
    """The vectors of a thread that the launched kernel has registers for reach the
    last pixel of the workgroup's part, for every width of a workgroup and every
    image of up to 4096 vectors, beyond which workgroups are large."""
    run_cpp(tmp_path, "cf_gnorm_plan.h", "gnorm", """
    bool small[2] = {false, false};
    for (int D = 8; D <= 4096; D += D < 520 ? 1 : 72)
        for (int64_t P = 1; P * ((D + 7) / 8) <= 4600; P++)
            for (int64_t groups : {1, 2, 100, 300, 3000})
                for (int most : {FORWARD_NV, BACKWARD_NV}) {
                    const int G = groups < 100 ? (int)groups : 4;
                    const Plan p = plan_of((groups + G - 1) / G, P, D * G, G, most, %d);
                    if (p.rows < 1)
                        continue;
                    const int has = held(p, most);
                    small[most == BACKWARD_NV] |= p.threads == 256 && p.nv > 8;
                    if (has < p.nv || (int64_t)has * p.rows < p.px || (p.threads == 256 && has > SMALL_NV)) {
                        printf("%%d channels a group, P %%lld, %%lld groups: %%d threads, nv %%d, held %%d\\n", D, (long long)P,
                               (long long)groups, p.threads, p.nv, has);
                        return 1;
                    }
                }
    if (!small[0] || !small[1])
        return 1;
    """ % cus)


def test_the_sizes_of_the_tile_tests_take_every_tile(tmp_path):
    """The tests of the tiles on the GPU (test_heads_gpu.py) run both behind each
    kind of product, and products over whole and split axes."""
    from test_heads_gpu import LARGE_GATED, LARGE_LINEAR

    products = []
    for r, C, H in LARGE_GATED:
        products += [("up", r, 2 * H, C, 1, "true", "MORE"), ("dh", r, H, C, 1, "true", "GATE"),
                     ("down", r, C, H, 1, "true", "STORE"), ("dx", r, C, 2 * H, 1, "true", "STORE"),
                     ("dw", C, H, r, 1, "true", "STORE"), ("dw", H, C, r, 2, "true", "STORE")]
    for r, C, V in LARGE_LINEAR:
        products += [("logits", r, V, C, 1, "true", "MORE"), ("dx of logits", r, C, V, 1, "true", "STORE"),
                     ("dw of logits", V, C, r, 1, "true", "STORE")]
    out = run_cpp(tmp_path, "cf_mm_plan.h", "mm", "".join(
        "{ const Plan p = plan_of(%d, %d, steps_of(%d), %d, %s, 256, %s); printf(\"%%d %%d\\n\", p.tile, p.splits); }\n"
        % q[1:] for q in products))
    seen = set()
    for q, line in zip(products, out.split("\n")):
        tile, splits = (int(v) for v in line.split())
        # behind a split sum of gates or logits the tile's own end does not run
        if splits == 1 or q[0] not in ("up", "dh", "logits"):
            seen.add((q[0], tile))
        seen |= {(tile, "split" if splits > 1 else "whole"), (q[0], "split" if splits > 1 else "whole")}
    missing = {(name, t) for name in ("up", "dh", "down", "dx", "dw", "logits") for t in range(2)} - seen
    missing |= {(name, "split") for name in ("up", "dh", "logits")} - seen
    assert not missing, missing
    assert {(t, k) for t in range(2) for k in ("split", "whole")} <= seen, seen
