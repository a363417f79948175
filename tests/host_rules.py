"""The library's host rules (which kernel, which variant a call gets), compiled from their headers for the tests."""
import functools
import os
import subprocess
import tempfile

from paper_2509_24014_b200 import build


@functools.lru_cache(maxsize=None)
def _program(header, expression, names):
    """A program that reads lines of whole numbers called `names` and prints the expression's value for each."""
    folder = tempfile.mkdtemp()
    main, exe = os.path.join(folder, "main.cc"), os.path.join(folder, "main")
    inputs = names.split()
    with open(main, "w") as f:
        f.write(f'#include <cstdio>\n#include "{header}"\nint main() {{ long long {", ".join(inputs)}; while (std::scanf("'
                + "%lld " * len(inputs) + '", ' + ", ".join("&" + x for x in inputs) + f") == {len(inputs)}) "
                f'std::printf("%lld\\n", static_cast<long long>({expression})); }}\n')
    subprocess.run(["g++", "-std=c++17", "-I", build.CSRC, main, "-o", exe], check=True)
    return exe


def evaluate(header, expression, names, rows):
    text = "".join(" ".join(str(int(x)) for x in row) + "\n" for row in rows)
    out = subprocess.run([_program(header, expression, names)], input=text, capture_output=True, text=True, check=True).stdout
    return [int(x) for x in out.split()]


def packed_is_pair(num_seqs, total_q, total_k, heads_q, heads_kv, causal):
    """Whether the rule sends a packed call to the CTA-pair kernel (no kernel is forced)."""
    if os.environ.get("SPARSED_PACKED_KERNEL"):
        return os.environ["SPARSED_PACKED_KERNEL"] == "pair"
    group = heads_q // heads_kv
    pack = max(d for d in range(1, group + 1) if group % d == 0 and 128 // d * d >= 124)
    return evaluate("dense_choice.h", "sparsed::packed_pair_pays(n, q, k, heads, tokens, causal != 0)",
                    "n q k heads tokens causal", [(num_seqs, total_q, total_k, heads_q // pack, 128 // pack, causal)]) == [1]
