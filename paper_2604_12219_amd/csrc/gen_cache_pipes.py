#!/usr/bin/env python3
"""Writes pasa_cache_pipes.hpp: the LDS-read + MFMA sequences of attention over the 4-bit cache (pasa_cache_tile.hip).

They are the ones of gen_mfma_pipes.py (whose helpers and register plan are used) but for the logits: keys and queries are fp16,
and one more matrix instruction per 32 keys adds what the groups' offsets contribute (see pasa_cache_tile.hip): its operands are
16 fp16 numbers a key, from LDS, and as many a query, in registers.  No tiles are requested: these kernels write their tiles themselves.

Run `python gen_cache_pipes.py` in this directory after changing it; the header is committed.
"""
import os

import gen_mfma_pipes as base
from gen_mfma_pipes import F, FS_O, FS_P0, FS_P1, FS_S0, FS_S1, FS_T, MFMA, NOP_AFTER, off, vr

MFMA_F16 = "v_mfma_f32_32x32x16_f16"
BIAS_ROW = 32  # bytes of a key's offset operands


class Pipe(base.LdsPipe):
    def issue(self, k, load):
        if load[0] == "b":  # offset operands of 32 keys
            self.lines.append(f"ds_read_b128 {F(k % self.nbuf)}, %[ab]{off(load[2] * 32 * BIAS_ROW)}")
            self.issued.append(1)
        else:
            super().issue(k, load)


def logits(D, half):
    acc = vr(FS_S0 if half == 0 else FS_S1, 16)
    return [dict(op=MFMA_F16, acc=acc, first=True, b="%[qb]", load=("b", 0, half))] + \
        [dict(op=MFMA_F16, acc=acc, first=False, b=f"%[q{st}]", load=("k", st, half)) for st in range(D // 16)]


def run(D, mf, before, after):
    lines = []
    pipe = Pipe(lines, D)
    pipe.k_addresses()
    n = len(mf)
    for k in range(min(pipe.nbuf, n)):
        pipe.issue(k, mf[k]["load"])
    for k in range(n):
        pipe.wait_for(k)
        lines += before.get(k, [])
        m = mf[k]
        lines.append(f"{m['op']} {m['acc']}, {F(k % pipe.nbuf)}, {m['b']}, {'0' if m['first'] else m['acc']}")
        if k + pipe.nbuf < n:
            pipe.issue(k + pipe.nbuf, mf[k + pipe.nbuf]["load"])
        lines += after.get(k, [])
    return lines + [NOP_AFTER]


def tile_step(D):
    """logits, online softmax and P V of one 64-key tile (fused_step of gen_mfma_pipes.py)"""
    nl, nt = D // 16 + 1, D // 32
    n_o = 16 * nt
    mf = logits(D, 0) + logits(D, 1)
    for half in range(2):
        for ks in range(2):
            for t in range(nt):
                mf.append(dict(op=MFMA, acc=vr(FS_O + 16 * t, 16), first=False, b=vr((FS_P0 if half == 0 else FS_P1) + 4 * ks, 4),
                               load=("v", 2 * half + ks, t)))
    after = {}
    pv0_end = 2 * nl + 2 * nt - 1
    base.spread(after, nl + 1, 2 * nl - 1, base.max_stream(FS_S0) + base.raise_max(n_o, True) + base.exp_stream(FS_S0, FS_P0))
    base.spread(after, 2 * nl + 1, pv0_end, base.max_stream(FS_S1) + base.raise_max(n_o, False) + base.exp_stream(FS_S1, FS_P1))
    after[pv0_end] += ["s_cmp_eq_u64 %[flag], 0", "s_cbranch_scc1 .Lfs_nors_%=", "s_nop 13"] + \
        [f"v_mul_f32 {vr(FS_O + i)}, {vr(FS_O + i)}, {vr(FS_T + 3)}" for i in range(n_o)] + [".Lfs_nors_%=:"]
    before = {2 * nl: ["s_nop 1"], 2 * nl + 2 * nt: ["s_nop 1"]}  # P^T / accumulators were written by VALU just before
    return run(D, mf, before, after)


def gen():
    out = ["// GENERATED by gen_cache_pipes.py -- do not edit.  LDS-read + MFMA sequences of attention over the 4-bit cache (gfx950), one asm\n"
           "// statement each; v168..v255 are theirs.\n"
           "#pragma once\n#include \"pasa_device.hpp\"\n\ntypedef _Float16 f16x8 __attribute__((ext_vector_type(8)));\n\nnamespace cache_pipes {\n\n"]
    for D in (128, 64):
        ns, nt = D // 16, D // 32
        qin = [f'[q{s}] "v"(q[{s}])' for s in range(ns)] + ['[qb] "v"(qb)']
        text = lambda lines: "\n".join(f'      "{l}\\n\\t"' for l in lines)
        clob = lambda regs, more: ", ".join([f'"v{r}"' for r in regs] + [f'"{c}"' for c in more])
        s_out = '"=&{v[168:183]}"(c0), "=&{v[184:199]}"(c1)'
        s_in = ", ".join(['[ak] "v"(ak)', '[ab] "v"(ab)'] + qin)
        out.append(f"// c0, c1 = logits of the tile's keys 0..31 and 32..63;  ak: K tile address + lane's row-fragment offset, ab: the same of its offset operands\n"
                   f"PASA_DEVICE void logits(uint32_t ak, uint32_t ab, const f16x8 (&q)[{ns}], f16x8 qb, f32x16& c0, f32x16& c1) {{\n"
                   f"  asm volatile(\n{text(run(D, logits(D, 0) + logits(D, 1), {}, {}))}\n      : {s_out}\n      : {s_in}\n"
                   f"      : {clob(range(200, 256), ['memory'])});\n}}\n\n")
        outs = base.o_ops(nt) + ['[m] "+v"(m)', '[l] "+v"(l)', '[flag] "=&s"(flag)']
        ins = ['[ak] "v"(ak)', '[ab] "v"(ab)', '[av0] "v"(av0)', '[av1] "v"(av1)', '[c] "v"(c)'] + qin
        out.append(f"// One whole 64-key tile against the wave's 32 queries: logits, online softmax, P V.  av0, av1: V tile address + the two column-fragment\n"
                   f"// offsets; m, l: running maximum (log2 units) and normaliser share; c: the lane's logit scale * log2(e)\n"
                   f"PASA_DEVICE void tile_step(uint32_t ak, uint32_t ab, uint32_t av0, uint32_t av1, const f16x8 (&q)[{ns}], f16x8 qb, f32x16 (&o)[{nt}], float& m,\n"
                   f"                           float& l, float c) {{\n  uint64_t flag;\n"
                   f"  asm volatile(\n{text(tile_step(D))}\n      : {', '.join(outs)}\n      : {', '.join(ins)}\n"
                   f"      : {clob(range(base.FUSED_CLOBBER_LO, 256), ['memory', 'scc', 'vcc'])});\n}}\n\n")
    out.append("}  // namespace cache_pipes\n")
    return "".join(out)


if __name__ == "__main__":
    here = os.path.dirname(os.path.abspath(__file__))
    with open(os.path.join(here, "pasa_cache_pipes.hpp"), "w") as f:
        f.write(gen())
