"""Calls of the selective scan whose token axis is cut, as keyword arguments of scan_util.Scan: run by tests on the GPU, and looked at on the CPU, where it shows whether they
are cut."""
D = 72
CUT = [dict(B=1, T=700), dict(lengths=[520, 1, 256, 0, 255], front=1), dict(lengths=[130, 128], longest=1000), dict(lengths=[3, 700, 40], front=1)]
STATES = (8, 16, 32, 64)
# more (sequence, channel block) units than a card has compute units, and one long sequence
MANY = dict(lengths=[600, 17, 40, 1, 0, 33, 5, 64, 9, 80, 2, 16, 31, 70, 12, 3, 28, 45, 100, 7], front=4, tail=3)
MANY_D = 1024


def sizes(call):
    """(B, T, rows; None without offsets)"""
    if "B" in call:
        return call["B"], call["T"], None
    lengths = call["lengths"]
    return len(lengths), call.get("longest", max(lengths)), call.get("front", 0) + sum(lengths) + call.get("tail", 0)
