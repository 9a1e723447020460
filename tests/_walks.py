"""The walk that a launch over packed prompts takes, by the launch's own rule (csrc/prompt_walk.h),
so that a test of a kernel says which of its forms it runs; tests/test_prompt_walk_cpu.py holds it
against the rule."""
TEAM4, TEAM8, SPLIT, HALVES = "four waves", "eight waves", "split keys", "two waves to a row"


def walk(Hq, Hkv, D, dtype, lens):
    """The walk of one launch (at most 128 sequences with tokens)."""
    bf16, group = dtype == "bf16", Hq // Hkv
    lens = [n for n in lens if n]
    assert lens and len(lens) <= 128
    units = sum((n * group + 31) // 32 for n in lens) * Hkv
    if not (bf16 and D == 256) and units <= (256 if bf16 and D == 128 else 1024):
        return SPLIT
    if units >= 4096:
        return TEAM8
    if not bf16:
        return HALVES
    longest, pairs = max(lens), sum(n * (n + 64) for n in lens)
    return HALVES if D < 256 and longest >= 512 and longest * 65536 * 5 > pairs * Hq * 6 else TEAM4
