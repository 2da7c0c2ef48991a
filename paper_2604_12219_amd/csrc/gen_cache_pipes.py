#!/usr/bin/env python3
"""Writes pasa_cache_pipes.hpp: the LDS-read + MFMA sequences of attention over the 4-bit cache (pasa_cache_tile.hip).

They are the ones of gen_mfma_pipes.py (whose helpers and register plan are used) but for the logits: keys and queries are fp16,
and one more matrix instruction per 32 keys adds what the groups' offsets contribute (see pasa_cache_tile.hip): its operands are
16 fp16 numbers a key, from LDS, and as many a query, in registers.  No tiles are requested: these kernels write their tiles themselves.

Run `python gen_cache_pipes.py` in this directory after changing it; the header is committed.
"""
import os

import gen_mfma_pipes as base
from gen_mfma_pipes import FS_P0, FS_P1, FS_S0, FS_S1, FS_T, MFMA, NOP_AFTER, Cold, F, exp_stream, max_stream, off, pending, pour, vr

MFMA_F16 = "v_mfma_f32_32x32x16_f16"
BIAS_ROW = 32  # bytes of a key's offset operands: 16 for each half-wave, those of a tile's 64 keys for the first one, then for the other


def growth(cold, flag, corr):
    """after max_stream: where the lane's maximum is larger than m, m <- that + 8, and l and the factor `corr` for the accumulators follow; `flag` is not zero
    then.  m so stands for a bound of the logits that they reach seldom: weights start at 2^-8 instead of 1 (to the same relative accuracy), and of the 64
    tiles of 4096 tokens a few change m, where an exact maximum makes one of a wave's 32 rows do so in most of them."""
    t0, t1, t2 = (vr(FS_T + i) for i in range(3))
    body = [f"v_mov_b32 {t1}, {t0}", "s_nop 1", f"v_permlane32_swap_b32 {t0}, {t1}", "s_nop 0",
            f"v_max_f32 {t0}, {t0}, {t1}", f"v_add_f32 {t1}, 0x41000000, {t0}", f"v_cmp_gt_f32 vcc, {t0}, %[m]", "s_nop 1",
            f"v_cndmask_b32 {t1}, %[m], {t1}, vcc", f"v_sub_f32 {t2}, %[m], {t1}", f"v_exp_f32 {corr}, {t2}",
            f"v_mov_b32 %[m], {t1}", "s_nop 0", f"v_mul_f32 %[l], %[l], {corr}"]
    return tuple([f"v_cmp_gt_f32 vcc, {t0}, %[m]", f"s_mov_b64 {flag}, vcc"] + cold.block("s_cbranch_vccnz", body))


def qk(D, half, tile=0):
    acc = vr(FS_S0 if half == 0 else FS_S1, 16)
    return [dict(op=MFMA_F16, acc=acc, first=True, b="%[qb]", load=("b", 0, half, tile))] + \
        [dict(op=MFMA_F16, acc=acc, first=False, b=f"%[q{st}]", load=("k", st, half, tile)) for st in range(D // 16)]


def pv(D, half, tile=0):
    return [dict(op=MFMA, **dict(m, load=(*m["load"], tile))) for m in base.pv_mfmas(D, half)]


CONV_R = 216                # v[216:219]: 8 converted values on their way to LDS
CONV_T = FS_T + 5           # three temporaries that the softmax streams leave alone


def convert(D, n, group):
    """n code words of K and of V, converted and written to the tiles `group` (keys8, values8 in pasa_cache_tile.hip)"""
    r, t = [vr(CONV_R + i) for i in range(4)], [vr(CONV_T + i) for i in range(3)]
    out = []

    def write(name, j, shift):
        addr = f"%[{name}]"
        if j:
            out.append(f"v_xor_b32 {t[0]}, {hex(j << shift)}, {addr}")
            addr = t[0]
        out.append(f"ds_write_b128 {addr}, {vr(CONV_R, 4)}{off(group * 2 * 128 * D)}")

    for j in range(n):
        for i in range(4):  # channels i and i + 4
            out.append(f"v_lshlrev_b32 {r[i]}, {6 - 4 * i}, %[kc{j}]" if i < 2 else f"v_lshrrev_b32 {r[i]}, {4 * i - 6}, %[kc{j}]")
            out.append(f"v_and_or_b32 {r[i]}, {r[i]}, %[mask], %[one]")
            out.append(f"v_pk_fma_f16 {r[i]}, {r[i]}, %[kf{j}], %[kf{j}] op_sel:[0,0,1] op_sel_hi:[1,0,1]")
        write("kst", j, 6)

    def mix(dst, src, hi, b):
        out.append(f"v_fma_mix_f32 {dst}, {src}, %[vs], %[vm{b}] op_sel:[{hi},0,0] op_sel_hi:[1,0,0]")

    for j in range(n):
        src = f"%[vc{j}]"
        for i in range(2):  # channels 2 i, 2 i + 1 -> r[i]; 2 i + 4, 2 i + 5 -> r[i + 2]
            out.append(f"v_and_or_b32 {t[1]}, {src}, %[high], %[c64]")
            out.append(f"v_and_or_b32 {t[0]}, {src}, %[low], %[c1024]")  # (src may be t[0])
            mix(r[i], t[0], 0, 0)
            mix(t[2], t[1], 0, 1)
            mix(r[i + 2], t[0], 1, 0)
            out.append(f"v_cvt_pk_bf16_f32 {r[i]}, {r[i]}, {t[2]}")
            mix(t[1], t[1], 1, 1)
            if i == 0:  # the upper half of every 16 bits
                out.append(f"v_lshrrev_b32 {t[0]}, 8, {src}")
                src = t[0]
            out.append(f"v_cvt_pk_bf16_f32 {r[i + 2]}, {r[i + 2]}, {t[1]}")
        write("vst", j, 4)
    return out


def run(D, mf, before, after, group=0, prologue=()):
    """MFMA k of `mf` with its operand fetch issued six MFMAs ahead (as pipe_run of gen_mfma_pipes.py), from a group of two tiles of the ring.
    LDS instructions end in order, so a wait counts those issued after the one it waits for."""
    lines, ends, count, nbuf = [], [], [0], 6

    def issue(k):
        f = k % nbuf
        kind, a, b, tile = mf[k]["load"]
        at = (2 * group + tile) * 128 * D
        if kind == "b":  # offset operands of 32 keys
            lines.append(f"ds_read_b128 {F(f)}, %[ab]{off((2 * group + tile) * 64 * BIAS_ROW + b * 32 * (BIAS_ROW // 2))}")
        elif kind == "k":
            lines.append(f"ds_read_b128 {F(f)}, %[ka{a}]{off(at + b * 64 * D)}")
        else:
            lines.append(f"ds_read_b64_tr_b16 {base.Flo(f)}, %[va{2 * b}]{off(at + a * 32 * D)}")
            lines.append(f"ds_read_b64_tr_b16 {base.Fhi(f)}, %[va{2 * b + 1}]{off(at + a * 32 * D)}")
        count[0] += 2 if kind == "v" else 1
        ends.append(count[0])

    n = len(mf)
    for k in range(min(nbuf, n)):
        issue(k)
    lines += list(prologue)
    for k in range(n):
        lines.append(f"s_waitcnt lgkmcnt({min(count[0] - ends[k], 15)})")
        lines += before.get(k, [])
        m = mf[k]
        lines.append(f"{m['op']} {m['acc']}, {F(k % nbuf)}, {m['b']}, {'0' if m['first'] else m['acc']}")
        if k + nbuf < n:
            issue(k + nbuf)
        lines += after.get(k, [])
        count[0] += sum(x.startswith("ds_") for x in after.get(k, []))
    return lines


def step_streams(after, n, at, n_o, cold):
    """what runs beside the n MFMAs (from number `at` on) of a step: logits of 32 keys -> S0, P V with P0, logits -> S1, P V with P1; meanwhile the softmax of
    what S1 held before -> P1 and of S0 -> P0 (the pipelined step of gen_mfma_pipes.py)"""
    corr1 = vr(FS_T + 3)
    late = {}
    late[1] = list(pending(cold, "%[flag]", "%[corr]", n_o, "s_nop 3"))  # left by the step before
    # (done with S1 before the MFMAs of the second half write it; S0 is long complete)
    first = [growth(cold, "%[flag1]", corr1)] + exp_stream(FS_S1, FS_P1)
    if at:  # the maximum of S1: at the start of the statement it has no MFMA to run beside
        first = max_stream(FS_S1) + first
    pour(late, n, first, first=0 if at else 1, end=0.5)
    pour(late, n, max_stream(FS_S0) + [growth(cold, "%[flag]", "%[corr]")] + exp_stream(FS_S0, FS_P0), begin=0.5)
    k = n // 2 + 1  # the P V of the first half is through
    late[k] = list(pending(cold, "%[flag1]", corr1, n_o, "s_nop 3")) + late.get(k, [])
    for k, x in late.items():
        after.setdefault(at + k, []).extend(x)


def pipe_steps(D, words, group, tiles):
    """for each of the tiles: P V of it, logits of the next one; its V is the tile of this number in the V group, the next one's K in the K group.
    words > 0: meanwhile the other groups are filled"""
    n_o = 16 * (D // 32)
    mf, after, text = [], {}, []
    for tile in range(tiles):
        part = qk(D, 0, tile) + pv(D, 0, tile) + qk(D, 1, tile) + pv(D, 1, tile)
        cold = Cold(f"ps{group}_{tile}_")
        step_streams(after, len(part), len(mf), n_o, cold)
        mf += part
        text.append(cold)
    if words:
        pour(after, len(mf), convert(D, words, 1 - group))
    return run(D, mf, {}, after, group, prologue=max_stream(FS_S1)) + sum([c.text() for c in text], [])


def pipe_start(D):
    """logits of a tile and the softmax of its first half"""
    mf = qk(D, 0) + qk(D, 1)
    n, q = len(mf), len(mf) // 2
    cold = Cold("pb")
    after = {}
    pour(after, n, max_stream(FS_S0) + [growth(cold, "%[flag]", "%[corr]")] + exp_stream(FS_S0, FS_P0), first=q + 1, begin=(q + 1) / n)
    return run(D, mf, {}, after) + [NOP_AFTER] + cold.text()


def pipe_end(D):
    """P V of the last tile and the softmax of its second half"""
    n_o = 16 * (D // 32)
    mf = pv(D, 0) + pv(D, 1)
    q = len(mf) // 2
    cold = Cold("pe")
    after = {}
    pour(after, q, [growth(cold, "%[flag]", "%[corr]")] + exp_stream(FS_S1, FS_P1))
    before = {q: list(pending(cold, "%[flag]", "%[corr]", n_o, NOP_AFTER)) + ["s_nop 1"]}
    return run(D, mf, before, after, prologue=list(pending(cold, "%[flag]", "%[corr]", n_o, NOP_AFTER)) + max_stream(FS_S1) + ["s_nop 1"]) + \
        [NOP_AFTER] + cold.text()


def gen():
    out = ["// GENERATED by gen_cache_pipes.py -- do not edit.  LDS-read + MFMA sequences of attention over the 4-bit cache (gfx950), one asm\n"
           "// statement each.\n"
           "#pragma once\n#include \"pasa_mfma_pipes.hpp\"\n\ntypedef _Float16 f16x8 __attribute__((ext_vector_type(8)));\n\nnamespace cache_pipes {\n\n"
           "using pipes::PipeState;\n\n"]
    s0, p1, rest = range(FS_S0, FS_S0 + 16), range(FS_P1, FS_P1 + 8), list(range(FS_T, 256))
    for D in (128, 64):
        ns, nt = D // 16, D // 32

        def emit(comment, head, pre, lines, outs, ins, clob):
            text = "\n".join(f'      "{l}\\n\\t"' for l in lines)
            # No "memory": the compiler's waits for loads in flight, those of spilled values among them, leave out the pinned registers of statements that
            # have it, and such a load can arrive on top of a result.  The ring's order is that of the barriers, which do say so.
            regs = ", ".join([f'"v{r}"' for r in clob] + ['"scc"', '"vcc"'])
            out.append(f"{comment}PASA_DEVICE void {head} {{\n{pre}  asm volatile(\n{text}\n      : {', '.join(outs)}\n      : {', '.join(ins)}\n"
                       f"      : {regs});\n}}\n\n")

        q_args = f"const f16x8 (&q)[{ns}], f16x8 qb"
        state = f"f32x16 (&o)[{nt}], float& m, float& l, PipeState& st"
        ml = ['[m] "+v"(m)', '[l] "+v"(l)']
        sb = '"+{v[184:199]}"(st.s1)'
        pa = [f'"+{{v[{200 + 4 * k}:{203 + 4 * k}]}}"(st.p0[{k}])' for k in range(2)]
        carry = ['[corr] "+v"(st.corr)', '[flag] "+s"(st.flag)']
        kin = [f'[ka{s}] "v"(ka[{s}])' for s in range(ns)] + ['[ab] "v"(ab)'] + [f'[q{s}] "v"(q[{s}])' for s in range(ns)] + ['[qb] "v"(qb)']
        vin = [f'[va{s}] "v"(va[{s}])' for s in range(2 * nt)]
        cin, group_in = ['[c] "v"(c)'], ['[par] "s"(group)']
        k_args = f"const uint32_t (&ka)[{ns}], uint32_t ab"
        v_args = f"const uint32_t (&va)[{2 * nt}]"
        emit("// c0, c1 = logits of keys 0..31 and 32..63 of a tile.  ka, ab: the lane's addresses of its row fragments and of its offset operands; q, qb: the\n"
             "// queries and what they multiply the offsets with\n",
             f"logits({k_args}, {q_args}, f32x16& c0, f32x16& c1)", "", run(D, qk(D, 0) + qk(D, 1), {}, {}) + [NOP_AFTER],
             ['"=&{v[168:183]}"(c0)', '"=&{v[184:199]}"(c1)'], kin, range(226, 256))
        emit("// Start of a run of pipelined steps: logits of a tile, softmax of its first half.  c: the lane's logit scale * log2(e); corr, flag of the\n"
             "// state are outputs\n",
             f"pipe_start({k_args}, {q_args}, float& m, float& l, float c, PipeState& st)", "", pipe_start(D),
             ml + ['"=&{v[184:199]}"(st.s1)'] + [x.replace("+", "=&") for x in pa] + ['[corr] "=&v"(st.corr)', '[flag] "=&s"(st.flag)'],
             kin + cin, list(s0) + list(p1) + rest)
        step_outs = base.o_ops(nt) + ml + [sb] + pa + carry + ['[flag1] "=&s"(flag1)']
        emit("// P V of a tile, logits of the next one.  va: the lane's addresses of the tile's column fragments; ka, ab: of the next tile's\n",
             f"pipe_step({k_args}, {v_args}, {q_args}, {state}, float c)", "  uint64_t flag1;\n", pipe_steps(D, 0, 0, 1), step_outs, kin + vin + cin,
             list(s0) + list(p1) + rest)
        words = D // 32
        conv = [f'[{x}{j}] "v"({x}[{j}])' for x in ("kc", "kf", "vc") for j in range(words)] + \
            [f'[{x}] "v"({x})' for x in ("vs", "vm0", "vm1", "kst", "vst")] + \
            [f'[{n}] "{c}"({v})' for n, c, v in (("mask", "v", "0x03c003c0u"), ("one", "s", "0x3c003c00u"), ("low", "v", "0x000f000fu"),
                                                 ("c1024", "s", "0x64006400u"), ("high", "v", "0x00f000f0u"), ("c64", "s", "0x54005400u"))]
        arr = f"const uint32_t (&%s)[{words}]"
        emit("// Two steps: P V of the two tiles of V group `group`, logits of the two of K group `group`, which are one tile further on; addresses are those of\n"
             f"// group 0.  Meanwhile {words} code words of K and of V are converted and written to the other groups: kc, vc the words, kf 16 s and\n"
             "// -24 s of a K word's group, times a power of two, as two fp16 numbers, vs, vm0, vm1 s, m - 1024 s and m - 64 s of the V words, kst, vst the lane's addresses\n",
             f"pipe_steps(int group, {k_args}, {v_args}, {q_args}, {state}, float c,\n"
             f"                            {arr % 'kc'}, {arr % 'kf'}, {arr % 'vc'}, float vs, float vm0, float vm1, uint32_t kst, uint32_t vst)",
             "  uint64_t flag1;\n", base.both_parities("ps", lambda group: pipe_steps(D, words, group, 2)), step_outs, kin + vin + cin + group_in + conv,
             list(s0) + list(p1) + list(range(CONV_R, CONV_R + 4)) + rest)
        emit("// End of a run: P V of the last tile\n", f"pipe_end({v_args}, {state}, float c)", "", pipe_end(D), base.o_ops(nt) + ml + [sb] + pa + carry,
             vin + cin, list(s0) + list(p1) + rest)
    out.append("}  // namespace cache_pipes\n")
    return "".join(out)


if __name__ == "__main__":
    here = os.path.dirname(os.path.abspath(__file__))
    with open(os.path.join(here, "pasa_cache_pipes.hpp"), "w") as f:
        f.write(gen())
