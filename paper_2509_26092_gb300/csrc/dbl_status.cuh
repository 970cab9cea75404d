// dbl_status.cuh -- the device-side status words of several files, read and cleared as one.  Host code alone.
#pragma once

#include "../../include/dbl.h"

namespace dbl {

struct StatusWord {
    int (*read)(int* status);  // DBL_OK or DBL_ERR_TIMEOUT
    int (*clear)();
};

// The first word that is set, all being cleared.  Every word is read before one is cleared, and only those that are set
// are: a call that fails leaves a timeout for the next to report.
inline int take_status_words(const StatusWord* words, int n, int* status)
{
    int first = DBL_OK, rc = DBL_OK;
    unsigned set = 0;
    for (int i = 0; i < n; ++i) {
        int v = DBL_OK;
        if ((rc = words[i].read(&v)) != DBL_OK) return rc;
        if (v != DBL_OK) set |= 1u << i;
        if (first == DBL_OK) first = v;
    }
    for (int i = 0; i < n; ++i)
        if ((set >> i & 1) && (rc = words[i].clear()) != DBL_OK) return rc;
    *status = first;
    return DBL_OK;
}

}  // namespace dbl
