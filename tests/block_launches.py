"""What the launches of a round of transformer-block operators (block_rounds.py) look like, on the CPU (not a test module)."""
import json
import os
import re
import subprocess
import sys
from collections import namedtuple

from block_rounds import CHILD, HERE
from paper_1902_04610_amd import build

# words: the first four that the kernel is given
Launch = namedtuple("Launch", "kernel grid block words")
SPLIT = 'return out + "====" + words().decode()'


def launches(rounds, tmp):
    """The Launches of each round, in order."""
    if not os.path.exists(build.LIB):
        build.build()
    libs = []
    for name in ("launch_words", "launch_recorder"):
        libs.append(os.path.join(str(tmp), "lib%s.so" % name))
        subprocess.check_call(["gcc", "-O1", "-fPIC", "-shared", "-Wall", "-o", libs[-1], os.path.join(HERE, name + ".c"), "-ldl"])
    child = CHILD.replace("up = lambda", "words = ctypes.CDLL(None).words_take\nwords.restype = ctypes.c_char_p\nup = lambda", 1)
    assert child.count("    pool.close()\n    return out\n") == 1
    child = child.replace("    pool.close()\n    return out\n", "    pool.close()\n    %s\n" % SPLIT)
    env = dict(os.environ, LD_PRELOAD=":".join(libs + list(filter(None, [os.environ.get("LD_PRELOAD")]))), PYTHONPATH=build.ROOT)
    r = subprocess.run([sys.executable, "-c", child], input=json.dumps(rounds), cwd=build.ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    out = []
    for log in json.loads(r.stdout.splitlines()[-1]):
        names, words = log.split("====")
        names = re.findall(r"^launch (\S+) (\d+) (\d+) ", names, re.M)
        words = [tuple(map(int, line.split())) for line in words.splitlines()]
        assert len(names) == len(words)
        out.append([Launch(n, int(g), int(b), w) for (n, g, b), w in zip(names, words)])
    plain = subprocess.run(["c++filt"], input="\n".join(l.kernel for o in out for l in o), stdout=subprocess.PIPE, text=True, check=True).stdout
    plain = iter(re.sub(r"\((salus::)?Epilogue\)", "E", plain).replace("salus::", "").replace("(anonymous namespace)::", "").replace("void ", "").splitlines())
    return [[l._replace(kernel=next(plain).rsplit("(", 1)[0]) for l in o] for o in out]
