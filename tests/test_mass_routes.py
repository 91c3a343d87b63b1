"""Which calls that add up weights keep the scores of attention, and which form them again."""
import test_more_sequence_launches as more

KEPT, FORMED = "attend_scores", "attend_tiles"


def test_where_scores_are_kept(tmp_path):
    def call(B, new, length, heads, dtype=0):
        return dict(more.BASE, entry="mass", B=B, T=B * new, rows=new, heads=heads, dtype=dtype, length=length, workspace=1 << 40)

    # microseconds, formed again and kept
    cases = [(call(2, 88, 88, (8, 8, 96)), KEPT),             # 40, 22
             (call(12, 34, 34, (8, 2, 128)), KEPT),           # 37, 16
             (call(48, 34, 34, (4, 4, 256)), KEPT),           # 55, 45
             (call(64, 64, 500, (1, 1, 256)), KEPT),          # as few rows as attend() takes so
             (call(1, 172, 292, (96, 12, 96)), FORMED),       # 78, 211
             (call(1, 155, 155, (64, 8, 96)), FORMED),        # 53, 126
             (call(26, 31, 6196, (32, 8, 256)), FORMED),      # 3128, 4655
             (call(18, 101, 1629, (12, 12, 256)), FORMED),    # 860, 1210
             (call(28, 180, 3118, (24, 12, 128)), FORMED),    # 3076, 5628
             (call(12, 88, 88, (12, 12, 64)), FORMED),        # 27, 32
             (call(12, 64, 64, (32, 8, 128), 2), FORMED)]     # 26, 48
    for (c, want), names in zip(cases, more._launches(tmp_path, [c for c, _ in cases])):
        assert more._kinds(names)[0] == want, (c, names)
